// C ABI of the norm of many gradients and of clipping them: argument checks and launches.  Declarations and contracts live in include/moe.h.
#include <hip/hip_runtime.h>

#include "grads.hpp"

using namespace moe;

static int check_tensors(const moe_tensor_t *t, int32_t n, bool outputs) {
    if (n < 0 || (n && !t)) return MOE_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        if (t[i].count < 0 || (t[i].dtype != MOE_DT_F32 && t[i].dtype != MOE_DT_BF16)) return MOE_ERR_INVALID_ARG;
        if (t[i].count > (int64_t)1 << 43) return MOE_ERR_UNSUPPORTED;  // (chunks of a launch are counted in 32 bits)
        if (!t[i].count) continue;
        const uintptr_t odd = t[i].dtype == MOE_DT_F32 ? 3 : 1;
        if (!t[i].in || ((uintptr_t)t[i].in & odd)) return MOE_ERR_INVALID_ARG;
        if (outputs && (!t[i].out || ((uintptr_t)t[i].out & odd))) return MOE_ERR_INVALID_ARG;
    }
    return MOE_OK;
}
static int64_t chunks_of(const moe_tensor_t &t) {
    const int64_t each = (int64_t)kThreads * kGradPieces * (t.dtype == MOE_DT_F32 ? 4 : 8);
    return (t.count + each - 1) / each;
}
// The next tensors that go into one launch; returns how many of `t` they are (those without a number among them).
static int fill(const moe_tensor_t *t, int n, GradArgs *a, unsigned *groups) {
    *a = GradArgs{};
    int64_t chunks = 0;
    int i = 0;
    for (; i < n && a->n < kGradTensors; ++i) {
        const int64_t c = chunks_of(t[i]);
        if (!c) continue;
        if (chunks + c > 0xffff0000ll) break;
        const int at = a->n++;
        a->in[at] = t[i].in, a->out[at] = t[i].out, a->count[at] = t[i].count;
        if (t[i].dtype == MOE_DT_F32) a->f32[at >> 5] |= 1 << (at & 31);
        a->end[at] = (u32)(chunks += c);
    }
    *groups = (unsigned)(chunks < kGradGroups ? chunks : kGradGroups);
    return i;
}

extern "C" {

size_t moe_grad_workspace_bytes(const moe_tensor_t *tensors, int32_t n) {
    if (check_tensors(tensors, n, false) != MOE_OK) return 0;
    size_t parts = 0;
    GradArgs a;
    unsigned groups;
    for (int i = 0; i < n; parts += groups) i += fill(tensors + i, n - i, &a, &groups);
    return (parts * sizeof(double) + 255) / 256 * 256 + (parts ? 0 : 256);
}

int moe_grad_norm(const moe_tensor_t *tensors, int32_t n, double *sum_squares, float *norm, void *workspace, void *stream) {
    const int rc = check_tensors(tensors, n, false);
    if (rc) return rc;
    if (!sum_squares || ((uintptr_t)sum_squares & 7)) return MOE_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255)) return MOE_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    double *parts = (double *)workspace;
    int done = 0;
    for (int i = 0; i < n;) {
        GradArgs a;
        unsigned groups;
        i += fill(tensors + i, n - i, &a, &groups);
        if (!groups) continue;
        a.parts = parts + done;
        hipLaunchKernelGGL(k_grad_squares, dim3(groups), dim3(kThreads), 0, st, a);
        if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
        done += (int)groups;
    }
    hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(kGradNormThreads), 0, st, (const double *)parts, done, sum_squares, norm);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_grad_clip(const moe_tensor_t *tensors, int32_t n, const double *sum_squares, float max_norm, void *stream) {
    const int rc = check_tensors(tensors, n, true);
    if (rc) return rc;
    if (!sum_squares || ((uintptr_t)sum_squares & 7) || !(max_norm >= 0.f)) return MOE_ERR_INVALID_ARG;
    for (int i = 0; i < n;) {
        GradArgs a;
        unsigned groups;
        i += fill(tensors + i, n - i, &a, &groups);
        if (!groups) continue;
        a.sum = sum_squares, a.max_norm = max_norm;
        hipLaunchKernelGGL(k_grad_clip, dim3(groups), dim3(kThreads), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
    }
    return MOE_OK;
}

}  // extern "C"
