// The training kernels on the CPU: fibres for the threads of a workgroup, barriers and wave exchanges that count arrivals, guarded
// buffers.  The device source is compiled into the same unit.
#include "train_emu.h"

#include <setjmp.h>
#include <sys/mman.h>
#include <ucontext.h>
#include <unistd.h>

#include <cstdio>
#include <cstdlib>
#include <deque>
#include <map>
#include <vector>

dim3 threadIdx, blockIdx, blockDim, gridDim;

namespace {

const size_t kStack = 128 * 1024;
struct Pending { char *dst; const char *src; };
struct Fibre {
    ucontext_t ctx;
    jmp_buf at;  // where it goes on once it has begun
    bool begun = false;
    char *stack = nullptr;
    bool done = false;
    std::deque<Pending> loads;
};
struct Wave {
    unsigned arrived = 0, generation = 0;
    char slot[64][64];
};
ucontext_t g_main;
jmp_buf g_back;
std::vector<Fibre *> g_fibres;
std::vector<Wave> g_waves;
unsigned g_cur, g_live, g_arrived, g_generation;
long g_errors = 0;
const char *g_lds = nullptr;
size_t g_lds_bytes = 0;
const std::function<void()> *g_body = nullptr;

void error(const char *what) {
    if (g_errors++ < 5) fprintf(stderr, "train_emu: %s (block %u, thread %u)\n", what, blockIdx.x, g_cur);
}
// (swapcontext only begins a fibre: it enters the kernel each time)
void yield() {
    if (!_setjmp(g_fibres[g_cur]->at)) _longjmp(g_back, 1);
}
void release() {
    if (g_live && g_arrived == g_live) {
        g_arrived = 0;
        g_generation++;
    }
}
void body_of_fibre() {
    (*g_body)();
    Fibre &f = *g_fibres[g_cur];
    if (!f.loads.empty()) error("a thread ended with loads to LDS under way");
    f.loads.clear();
    f.done = true;
    g_live--;
    release();
    _longjmp(g_back, 1);
}
// all 64 lanes of the wave are here
void wave_sync() {
    Wave &w = g_waves[g_cur / 64];
    const unsigned g = w.generation;
    if (++w.arrived == 64) {
        w.arrived = 0;
        w.generation++;
    } else
        while (w.generation == g) yield();
}
template <class T> void put(const T &v) { memcpy(g_waves[g_cur / 64].slot[g_cur % 64], &v, sizeof(T)); }
template <class T> void put(const T &v, size_t at) { memcpy(g_waves[g_cur / 64].slot[g_cur % 64] + at, &v, sizeof(T)); }
template <class T> T get(unsigned lane, size_t at = 0) { T v; memcpy(&v, g_waves[g_cur / 64].slot[lane] + at, sizeof(T)); return v; }

std::map<void *, std::pair<void *, size_t>> g_maps;

}  // namespace

namespace emu {

void sync() {
    const unsigned g = g_generation;
    g_arrived++;
    release();
    while (g_generation == g) yield();
}

void launch(dim3 grid, dim3 block, const std::function<void()> &body) {
    const unsigned nt = block.x;
    while (g_fibres.size() < nt) {
        g_fibres.push_back(new Fibre);
        g_fibres.back()->stack = (char *)malloc(kStack);
    }
    g_waves.assign((nt + 63) / 64, Wave());
    g_body = &body;
    gridDim = grid;
    blockDim = block;
    for (unsigned by = 0; by < grid.y; by++)
        for (unsigned bx = 0; bx < grid.x; bx++) {
            blockIdx = dim3(bx, by, 0);
            g_live = nt;
            g_arrived = 0;
            for (unsigned t = 0; t < nt; t++) {
                Fibre &f = *g_fibres[t];
                getcontext(&f.ctx);
                f.ctx.uc_stack.ss_sp = f.stack;
                f.ctx.uc_stack.ss_size = kStack;
                f.ctx.uc_link = &g_main;
                f.done = f.begun = false;
                makecontext(&f.ctx, body_of_fibre, 0);
            }
            while (g_live)
                for (volatile unsigned t = 0; t < nt; t = t + 1) {
                    if (g_fibres[t]->done) continue;
                    g_cur = t;
                    threadIdx = dim3(t, 0, 0);
                    if (_setjmp(g_back)) continue;
                    Fibre &f = *g_fibres[t];
                    if (f.begun) _longjmp(f.at, 1);
                    f.begun = true;
                    setcontext(&f.ctx);
                }
        }
}

void *guarded_alloc(size_t bytes) {
    const size_t page = (size_t)sysconf(_SC_PAGESIZE);
    size_t body = (bytes + page - 1) / page * page;
    if (body == 0) body = page;
    char *base = (char *)mmap(nullptr, body + 2 * page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (base == (char *)MAP_FAILED) return nullptr;
    mprotect(base, page, PROT_NONE);
    mprotect(base + page + body, page, PROT_NONE);
    char *user = base + page + (body - (bytes + 15) / 16 * 16);  // the end against the guard page
    g_maps[user] = std::make_pair((void *)base, body + 2 * page);
    return user;
}
void guarded_free(void *p) {
    auto it = g_maps.find(p);
    if (it == g_maps.end()) return;
    munmap(it->second.first, it->second.second);
    g_maps.erase(it);
}

}  // namespace emu

void emu_lds_range(const char *base, size_t bytes) {
    g_lds = base;
    g_lds_bytes = bytes;
}
const char *emu_lds_check(const char *p, size_t bytes) {
    if (p < g_lds || p + bytes > g_lds + g_lds_bytes) {
        error("LDS access outside the array");
        return g_lds;
    }
    return p;
}
void emu_load_to_lds(uintptr_t lds, unsigned offset, emu_u32x4 d) {
    char *dst = (char *)emu_lds_check((const char *)lds + 16 * (g_cur % 64), 16);
    const char *base = (const char *)((uintptr_t)d[0] | (uintptr_t)d[1] << 32);
    g_fibres[g_cur]->loads.push_back(Pending{dst, offset < d[2] ? base + offset : nullptr});
}
void emu_wait_loads(int newest) {
    std::deque<Pending> &q = g_fibres[g_cur]->loads;
    while ((int)q.size() > newest) {
        if (q.front().src) memcpy(q.front().dst, q.front().src, 16);
        else memset(q.front().dst, 0, 16);
        q.pop_front();
    }
}

template <class V, int N> static emu_f32x4 mfma(V first, V second, emu_f32x4 c) {
    put(first, 0);
    put(second, 32);
    wave_sync();
    const unsigned lane = g_cur % 64, col = lane % 16, g = lane / 16;
    for (unsigned r = 0; r < 4; r++)
        for (unsigned q = 0; q < 4; q++) {
            const V x = get<V>(16 * q + 4 * g + r, 0), y = get<V>(16 * q + col, 32);
            for (int e = 0; e < N; e++) {
                if constexpr (N == 1) c[r] += x * y;
                else c[r] += (float)x[e] * (float)y[e];
            }
        }
    wave_sync();
    return c;
}
emu_f32x4 emu_mfma_bf16(emu_bf16x8 a, emu_bf16x8 b, emu_f32x4 c) { return mfma<emu_bf16x8, 8>(a, b, c); }
emu_f32x4 emu_mfma_f16(emu_f16x8 a, emu_f16x8 b, emu_f32x4 c) { return mfma<emu_f16x8, 8>(a, b, c); }
emu_f32x4 emu_mfma_f32(float a, float b, emu_f32x4 c) { return mfma<float, 1>(a, b, c); }
emu_s16x4 emu_read_transposed(const char *p) {
    emu_s16x4 v;
    memcpy(&v, p, 8);
    put(v);
    wave_sync();
    const unsigned lane = g_cur % 64, group = lane & ~15u, i = lane & 15;
    emu_s16x4 out;
    for (unsigned j = 0; j < 4; j++) out[j] = get<emu_s16x4>(group + 4 * j + i / 4)[i % 4];
    wave_sync();
    return out;
}
unsigned emu_wave_max(unsigned v) {
    put(v);
    wave_sync();
    unsigned m = 0;
    for (unsigned l = 0; l < 64; l++) m = get<unsigned>(l) > m ? get<unsigned>(l) : m;
    wave_sync();
    return m;
}

float emu_lanes_sum(float x, int lanes) {
    for (int by = 1; by < lanes; by *= 2) {
        put(x);
        wave_sync();
        const float y = get<float>((g_cur % 64) ^ by);
        wave_sync();
        x += y;
    }
    return x;
}

float emu_code_to_float(unsigned c) { return (float)((int)(c << 28) >> 28) / 16.0f; }
emu_u32x4 emu_exchange_words(emu_u32x4 w) {
    put(w);
    wave_sync();
    const unsigned lane = g_cur % 64;
    emu_u32x4 o;
    for (unsigned s = 0; s < 4; s++) o[s] = get<emu_u32x4>(16 * s + lane % 16)[lane / 16];
    wave_sync();
    return o;
}

void emu_wave_fence() { wave_sync(); }

extern "C" void *emu_alloc(size_t bytes) { return emu::guarded_alloc(bytes); }
extern "C" void emu_free(void *p) { emu::guarded_free(p); }
extern "C" long emu_errors() { return g_errors; }

// how many tiles are enough for the larger shapes: tests take them at small sizes
static int g_enough = 192;
extern "C" void emu_enough_tiles(int n) { g_enough = n; }
#define TG_ENOUGH_TILES g_enough
static unsigned g_copy_blocks = 1u << 23;
extern "C" void emu_copy_blocks(unsigned n) { g_copy_blocks = n; }
#define TG_COPY_BLOCKS g_copy_blocks
static size_t g_small = (size_t)-1;  // matrices that take one workgroup: bytes of its LDS at most
extern "C" void emu_series_small(size_t bytes) { g_small = bytes; }
#define TS_SMALL_MOST (g_small < TS_SMALL_LDS ? g_small : (size_t)TS_SMALL_LDS)
static int g_tile = -1;  // of the large ones: 0, 1, or as the rule says
extern "C" void emu_series_tile(int n) { g_tile = n; }
#define TS_TILE(rule) (g_tile >= 0 ? g_tile : (rule))
#include "../../paper_1911_11377_amd/csrc/train_device.hip"
#include "../../paper_1911_11377_amd/csrc/norm_device.hip"
#include "../../paper_1911_11377_amd/csrc/muon_device.hip"
#include "../../paper_1911_11377_amd/csrc/low_device.hip"

// a context that the training operators accept: they use nothing of its ring
extern "C" ckksmi_ctx *emu_train_context() {
    ckksmi_ctx *c = new ckksmi_ctx;
    c->device = 0;
    return c;
}
extern "C" void emu_train_context_free(ckksmi_ctx *c) { delete c; }

// what the k axes in parts take of the workspace at this number of rows, largest launch of a pass
extern "C" size_t emu_split_need(const ckksmi_gated_ff *f, int backward) {
    const FF d(*f);
    const Matrix none{nullptr, 0};
    auto launch = [&](std::vector<GemmProblem> p, bool gate) {
        const int splits = choose(p.data(), (int)p.size(), gate, d.es).splits;
        size_t sum = 0;
        for (const GemmProblem &q : p) sum += round_up(part_bytes(q, splits, gate), 256);
        return sum;
    };
    if (!backward) return std::max(launch({product(none, none, d.M, d.H, d.K)}, true), launch({product(none, none, d.M, d.O, d.H)}, false));
    GemmProblem dx = product(none, none, d.M, d.K, d.H), dw = product(none, none, d.H, d.K, d.M), down = product(none, none, d.O, d.H, d.M);
    dx.nsrc = 2;
    dw.nsrc = down.nsrc = d.sources(f->dtype);
    return std::max(launch({dw, dw, down}, false), std::max(launch({product(none, none, d.M, d.H, d.O)}, false), launch({dx}, false)));
}
// ... and what the workspace has for them
extern "C" size_t emu_split_room(const ckksmi_gated_ff *f, int backward) { return split_bytes(*f, backward); }
