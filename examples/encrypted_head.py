"""A gated head from training to encrypted answers: features with a label that no linear head can tell (the sign of a product),
trained in the clear with the activation that the encrypted side evaluates, then evaluated on encrypted features.

    python examples/encrypted_head.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1911_11377_amd import ckksmi, head  # noqa: E402


def features(rows, d_in, seed):
    """rows of uniform features (the last one 1: the head has no biases) and two targets, +-1 by the sign of x0 * x1 and by that of x2"""
    g = np.random.default_rng(seed)
    x = g.uniform(-1, 1, (rows, d_in))
    x[:, -1] = 1.0
    return x, np.stack([np.sign(x[:, 0] * x[:, 1]), np.sign(x[:, 2])], axis=1)


def train(ctx, device, act, dtype, d_in=8, d_hidden=16, rows=256, steps=300, lr=0.02, seed=1):
    """the trained weights (float32 arrays) and the loss at the first and the last step"""
    g = torch.Generator().manual_seed(seed)
    weights = [(torch.randn(s, generator=g) * s[1] ** -0.5).to(device) for s in ((d_hidden, d_in), (d_hidden, d_in), (2, d_hidden))]
    h = head.GatedHead(ctx, rows, weights, act, dtype, lambda shape, t: torch.zeros(shape, dtype=t, device=device))
    first = last = None
    for t in range(steps):
        x, target = (torch.from_numpy(a).to(device) for a in features(rows, d_in, 1000 + t % 16))
        target = target.float()

        def loss(y, dy):
            off = y.float() - target
            dy.copy_(off * (2.0 / off.numel()))
            return off.square().mean()

        value = h.step(x.to(dtype), loss, lr * (1 - t / steps))
        first, last = value if t == 0 else first, value
    return [w.cpu().numpy() for w in weights], float(first), float(last)


def clear(weights, act, x):
    """the head in 64 bits"""
    from paper_1911_11377_amd.training import CUBICS

    g, u = x @ weights[0].T.astype(np.float64), x @ weights[1].T.astype(np.float64)
    return (sum(c * g**k for k, c in enumerate(CUBICS[act])) * u) @ weights[2].T.astype(np.float64)


def encrypted(ctx, weights, act, x, to_dev, empty, to_host, workspace, stream=None, scale=2.0**45, seed=7):
    """answers for the rows of x (one a slot) through encryption, the head on ciphertexts, and decryption"""
    N, level = ctx.N, ctx.n_q
    rows, d_in = x.shape
    # client: keys and one ciphertext a feature
    s = ctx.sample_ternary(seed)
    pk = ctx.keygen_public(s, ctx.sample_uniform(seed + 1, list(range(ctx.n_q))), ctx.sample_error(seed + 2))
    rlk_a = np.stack([ctx.sample_uniform(seed + 10 + j, list(range(ctx.T))) for j in range(ctx.beta_top)])
    rlk = ctx.keygen_relin(s, rlk_a, np.stack([ctx.sample_error(seed + 100 + j) for j in range(ctx.beta_top)]))
    cts = []
    for f in range(d_in):
        slots = np.zeros(N // 2)
        slots[:rows] = x[:, f]
        small = [ctx.sample_ternary(seed + 1000 + 3 * f), ctx.sample_error(seed + 1001 + 3 * f), ctx.sample_error(seed + 1002 + 3 * f)]
        cts.append(ctx.encrypt(pk, ctx.encode(slots, scale, level), *small, level))
    # server: weights in the clear, features encrypted
    p = head.plan(*weights, act, ctx.q, level, scale)
    ws = workspace(head.workspace_bytes(ctx, p, max_items=8))
    y = head.forward(ctx, p, to_dev(np.stack(cts)), to_dev(rlk), empty, to_dev, ws, stream=stream, max_items=8)
    # client
    out = to_host(y).reshape(p.d_out, 2, p.level_out, N)
    return np.stack([ctx.decode(ctx.decrypt(s, out[o], p.level_out), p.level_out, p.scale_out).real[:rows] for o in range(p.d_out)], axis=1)


def main():
    device, act = "cuda:0", "square"
    ctx = ckksmi.Context(13, 6, 50, 1, 51, 1, device=0)
    weights, first, last = train(ctx, device, act, torch.bfloat16)
    print("training loss %.3f -> %.3f" % (first, last))

    def to_dev(a):
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).to(device)

    def empty(*shape):
        return torch.empty(shape, dtype=torch.int64, device=device)

    x, target = features(1024, 8, 5)
    got = encrypted(ctx, weights, act, x, to_dev, empty, lambda t: t.cpu().numpy().view(np.uint64), lambda n: empty(max(1, n // 8)))
    want = clear(weights, act, x)
    print("1024 encrypted answers: off by at most %.2g; labels right %.1f %% and %.1f %%" % (
        np.abs(got - want).max(), *(100.0 * np.mean(np.sign(got) == target, axis=0))))


if __name__ == "__main__":
    main()
