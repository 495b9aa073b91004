// What the entry points of include/ckksmi_train.h share on the host: limits, checks of pointers, workspaces.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstring>

#include "device_call.h"
#include "../../include/ckksmi_train.h"

namespace {

constexpr int64_t kMaxDim = 1 << 20, kMaxRows = 0x7fffffff - 256;
constexpr double kMaxThreads = 4294967295.0;  // of a launch, along x
constexpr int kMaxBlocks = (1 << 24) - 1;      // workgroups of 256 threads

inline size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline bool dtype_ok(int d) { return d == CKKSMI_F32 || d == CKKSMI_BF16 || d == CKKSMI_F16; }

// [a, a + na) and [b, b + nb) share a byte
inline bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    if (!a || !b || !na || !nb) return false;
    const char *x = (const char *)a, *y = (const char *)b;
    return x < y + nb && y < x + na;
}

// A workspace handed out piece by piece (workspace_of() has counted the pieces)
struct Carve {
    char *base;
    size_t used = 0;
    explicit Carve(void *p) : base((char *)p) {}
    char *take(size_t bytes) {
        char *p = base + used;
        used += round_up(bytes, 256);
        return p;
    }
};

}  // namespace
