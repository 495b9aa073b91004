"""Plans of training.py and head.py on the CPU stand-in: what they refuse, what they ask for and what a call is given."""
import math

import pytest
import torch

import train_emu_support as emu
from paper_1911_11377_amd import training

pytestmark = pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = emu.EmuContext()
    yield c
    assert c.errors() == 0
    c.close()


class Calls:
    """a context that counts the calls and makes none"""

    _h = None

    def __init__(self):
        self.made = []

    def _call(self, name, *args):
        self.made.append(name)

    @staticmethod
    def _stream(stream):
        return None


@pytest.mark.parametrize("width", [1, 8])
@pytest.mark.parametrize("which", ["x", "y", "dy", "dx"])
def test_rows_that_lie_on_each_other_are_refused(which, width):
    """a row repeated by expand() and rows closer than their width: a distance of 0 means dense rows to the library"""
    rows = 5
    ff = training.GatedFF(Calls(), width, 16, width, F32, "square")
    w = [torch.zeros(16, width), torch.zeros(16, width), torch.zeros(width, 16)]
    dw = [torch.zeros_like(t) for t in w]
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    overlapping = [torch.zeros(1, width).expand(rows, width)]
    if width > 1:
        overlapping.append(torch.zeros(64).as_strided((rows, width), (width - 1, 1)))
    for bad in overlapping:
        t = {k: torch.zeros(rows, width) for k in ("x", "y", "dy", "dx")}
        t[which] = bad
        with pytest.raises(ValueError):
            ff.forward(t["x"], *w, t["y"], room)
            ff.backward(t["x"], *w, room, t["dy"], t["dx"], *dw, room)
    # one row has no distance, and rows further apart are taken as they are
    ff.forward(torch.zeros(1, width).expand(1, width), *w, torch.zeros(1, width), room)
    ff.forward(torch.zeros(rows, width + 3)[:, :width], *w, torch.zeros(rows, width), room)
