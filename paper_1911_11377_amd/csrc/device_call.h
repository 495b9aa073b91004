// What every device entry point uses: kernel launches with their timing, error recording, stream and context checks.
#pragma once
#ifndef CKKSMI_EMULATE
#include <hip/hip_runtime.h>
#define CKKSMI_LAUNCH(kern, grid, block, stream, ...) hipLaunchKernelGGL(kern, grid, block, 0, stream, __VA_ARGS__)
#endif

#include "ckksmi_internal.h"

// Launch `kern`; when profiling is on, bracket it with two events on the same stream and
// remember them under kernel class `kid` together with `units` of algorithmic work.
#define KL(c, kid, units, kern, grid, block, st, ...)                                   \
    do {                                                                                \
        ProfRec *pr_ = (c)->prof_on ? prof_begin((c), (kid), (double)(units), (st)) : nullptr; \
        CKKSMI_LAUNCH(kern, grid, block, st, __VA_ARGS__);                              \
        if (pr_) (void)hipEventRecord((hipEvent_t)pr_->stop, (st));                     \
    } while (0)

// ... one of two instances of a kernel template
#define KL2(c, kid, units, first, kern1, kern2, grid, block, st, ...)              \
    do {                                                                            \
        if (first) KL(c, kid, units, kern1, grid, block, st, __VA_ARGS__);          \
        else KL(c, kid, units, kern2, grid, block, st, __VA_ARGS__);                \
    } while (0)

namespace {

ProfRec *prof_begin(ckksmi_ctx *c, int kid, double units, hipStream_t st) {
    hipEvent_t a, b;
    if (hipEventCreate(&a) != hipSuccess) return nullptr;
    if (hipEventCreate(&b) != hipSuccess) { (void)hipEventDestroy(a); return nullptr; }
    (void)hipEventRecord(a, st);
    c->prof.push_back(ProfRec{kid, units, (void *)a, (void *)b});
    return &c->prof.back();
}

struct Guard {  // records the first HIP error of a call
    ckksmi_ctx *c;
    bool ok = true;
    explicit Guard(ckksmi_ctx *ctx) : c(ctx) {}
    void check(hipError_t e) {
        if (e != hipSuccess && ok) { ok = false; c->last_hip_error = (int)e; }
    }
    int rc() {
        check(hipGetLastError());
        if (c->no_kernel.exchange(false)) return CKKSMI_EUNSUPPORTED;
        return ok ? CKKSMI_OK : CKKSMI_EDEVICE;
    }
};

inline bool dev_ok(const ckksmi_ctx *c) { return c && c->device >= 0; }
inline hipStream_t S(void *s) { return (hipStream_t)s; }

}  // namespace
