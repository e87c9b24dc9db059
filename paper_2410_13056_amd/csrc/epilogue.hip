// The epilogue by itself, for products whose outputs are in memory (those in mixed precision give fp32).  Eight values a
// lane and step, nothing shared: bound by bytes.
#include "epilogue.h"

namespace {

constexpr int kThreads = 256;

__global__ __launch_bounds__(kThreads) void epilogue_kernel(cmpq_epilogue_job a, int64_t groups) {
#pragma clang fp contract(off)
    const int64_t columns = (a.d + 7) / 8;
    for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < groups; at += (int64_t)gridDim.x * kThreads) {
        const int64_t t = at / columns, o = (at - t * columns) * 8;
        const int n = (int)min(a.d - o, (int64_t)8);
        Raw8 y, u, r, b, c;
        y.load(a.Y.ptr, a.Y.dtype, t * a.Y.ld + o, n);
        if (a.times.ptr) u.load(a.times.ptr, a.times.dtype, t * a.times.ld + o, n);
        if (a.residual.ptr) r.load(a.residual.ptr, a.residual.dtype, t * a.residual.ld + o, n);
        if (a.bias.ptr) b.load(a.bias.ptr, a.bias.dtype, o, n);
        if (a.times_bias.ptr) c.load(a.times_bias.ptr, a.times_bias.dtype, o, n);
        float v[8], x[8];
        y.values(a.Y.dtype, v);
        if (a.bias.ptr) {
            b.values(a.bias.dtype, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        activate(a.activation, v);
        if (a.times.ptr) {
            u.values(a.times.dtype, x);
            if (a.times_bias.ptr) {
                float z[8];
                c.values(a.times_bias.dtype, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] += z[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= x[i];
        }
        if (a.residual.ptr) {
            r.values(a.residual.dtype, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        store_some<8>(a.out.ptr, a.out.dtype, t * a.out.ld + o, n, v);
    }
}

}  // namespace

extern "C" int cmpq_epilogue(const cmpq_epilogue_job *j, void *stream) {
    if (!j || j->m < 0 || j->d < 0 || !known_activation(j->activation)) return CMPQ_EINVAL;
    const cmpq_rows in[] = {j->Y, j->bias, j->times, j->times_bias, j->residual, j->out};
    for (const cmpq_rows &a : in)
        if (a.ptr && !serving_dtype(a.dtype)) return CMPQ_EINVAL;
    if (j->times_bias.ptr && !j->times.ptr) return CMPQ_EINVAL;
    if (j->m == 0 || j->d == 0) return CMPQ_OK;
    if (!j->Y.ptr || !j->out.ptr) return CMPQ_EINVAL;
    if (j->Y.ld < j->d || j->out.ld < j->d || (j->times.ptr && j->times.ld < j->d) || (j->residual.ptr && j->residual.ld < j->d)) return CMPQ_ESHAPE;
    if (j->m >= (1 << 24) || j->d >= (1 << 24)) return CMPQ_ESHAPE;
    const int64_t groups = j->m * cdiv(j->d, 8), blocks = cdiv(groups, kThreads);
    epilogue_kernel<<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), kThreads, 0, static_cast<hipStream_t>(stream)>>>(*j, groups);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
