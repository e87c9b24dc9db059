// Root-mean-square norm of a stream, or of two streams' sum, given as values or as rows in 8 bits.
// A workgroup a row, which stays in registers between its sum of squares and its outputs.  The squares are summed in 64
// bits, in an order that depends on the row's length alone, so a row's bits are the same in any batch and form.  Another
// order (a definition's, summed one by one) gives the same root but for a row in a hundred million or so, whose root lies
// within the sum's last bits of the middle between two numbers of fp32.
//
// Bound.  Many rows: by bytes.  4096 rows of 8192 in bfloat16 with their sum, 268 MB, 42.6 us (6.3 TB/s, what caches keep between
// calls included), as rows in 8 bits 42; where an fp32 stream is added 59 and 72.  One row: by what comes one after the other
// (the loads, the sum over the lanes, the root, the largest magnitude), 3.3 us, of rows in 8 bits 4.4.  Kernels for one type of all
// tensors are 10 to 20 % faster than the one that looks at each tensor's: 64 coded rows of 4096 4.2 us and 5.2.
#include "epilogue.h"
#include "int8_rows.h"

namespace {

constexpr int kAny = -1;

template <int N>
__device__ __forceinline__ void round_to(int dtype, float (&x)[N]) {
    if (dtype == CMPQ_F32) return;
    with_dtype(dtype, [&](auto like) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)(decltype(like))x[i];
    });
}

// Sum of the wavefronts' parts, the same in every lane: a tree whose two sides only change places from lane to lane.
template <int N>
__device__ __forceinline__ double total(const double *parts) {
    static_assert(N == 4 || N == 16, "wavefronts");
    if (N == 4) return (parts[0] + parts[1]) + (parts[2] + parts[3]);
    double v = parts[threadIdx.x & 15];
    const auto turn = [](double x, auto by) {
        const uint64_t u = (uint64_t)__double_as_longlong(x);
        return join_f64(row_turn<by()>((uint32_t)u), row_turn<by()>((uint32_t)(u >> 32)));
    };
    v += turn(v, std::integral_constant<int, 8>());
    v += turn(v, std::integral_constant<int, 4>());
    v += turn(v, std::integral_constant<int, 2>());
    return v + turn(v, std::integral_constant<int, 1>());
}

// Four sums over the wavefront for little more than one: lanes 16 q have that of v[0], v[2], v[1], v[3] (q = 0 .. 3), added in the
// order of wave_sum_f64.
__device__ __forceinline__ double wave_sums_f64(const double (&v)[4]) {
    const auto halves = [](double x, double y) {
        const uint64_t a = (uint64_t)__double_as_longlong(x), b = (uint64_t)__double_as_longlong(y);
        const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)a, (uint32_t)b, false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(a >> 32), (uint32_t)(b >> 32), false, false);
        return join_f64(lo[0], hi[0]) + join_f64(lo[1], hi[1]);
    };
    const uint64_t a = (uint64_t)__double_as_longlong(halves(v[0], v[1])), b = (uint64_t)__double_as_longlong(halves(v[2], v[3]));
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)a, (uint32_t)b, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(a >> 32), (uint32_t)(b >> 32), false, false);
    double x = join_f64(lo[0], hi[0]) + join_f64(lo[1], hi[1]);
    x += row_up_f64<8>(x);
    x += row_up_f64<4>(x);
    x += row_up_f64<2>(x);
    return x + row_up_f64<1>(x);
}

// 1 / sqrt(x) to about a step of fp64, rounded to fp32: the instruction's 26 bits, doubled twice by Newton's method.
__device__ __forceinline__ float one_over_root(double x) {
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = fma(r * 0.5, fma(-x * r, r, 1.0), r);
    return (float)r;
}

// KEPT steps of THREADS * 8 values hold the row; 0: it is read again for each pass.  TYPE: that of all tensors, or kAny.
template <int THREADS, int KEPT, bool CODED, int TYPE>
__global__ __launch_bounds__(THREADS) void rms_norm_kernel(cmpq_norm_job a, double per_value) {
#pragma clang fp contract(off)
    constexpr int kWaves = THREADS / 64, kStep = THREADS * 8, kHeld = KEPT > 0 ? KEPT : 1;
    // The sum's parts are those of 16 wavefronts with a step each, in their order, where rows in 8 bits may have either kernel.
    constexpr bool kApart = kWaves == 4 && KEPT > 2;
    static_assert(!kApart || KEPT <= 4, "steps");
    __shared__ double sums[kApart ? 16 : kWaves];
    __shared__ float most[kWaves];
    const int64_t row = CODED ? die_order(blockIdx.x, gridDim.x) : (int64_t)blockIdx.x;
    const auto type = [](int dtype) { return TYPE == kAny ? dtype : TYPE; };
    const int d = (int)a.d, first = threadIdx.x * 8;
    const int whole = CODED ? (int)pieces_deep(d) * kDepth : d;  // what is written of a row
    uint8_t *codes = nullptr;
    if (CODED) {
        codes = reinterpret_cast<uint8_t *>(a.codes) + row / kRows * pieces_deep(d) * kPiece + row % kRows * 16;
        if (row >= a.m) {  // rows that fill up the last piece
            for (int i = first; i < whole; i += kStep)
                *reinterpret_cast<uint2 *>(codes + i / kDepth * kPiece + i % kDepth / 16 * 256 + i % 16) = make_uint2(0, 0);
            return;
        }
    }
    float x[kHeld][8];
    Raw8 gain[kHeld];
    // s = x + a, rounded to its type.  `sum_is_there`: it has been written.
    auto load = [&](int i, float (&s)[8], bool sum_is_there) {
        const int n = min(max(d - i, 0), 8);
        Raw8 p, q;
        if (sum_is_there) {
            p.load(a.S.ptr, type(a.S.dtype), row * a.S.ld + i, n);
            p.values(type(a.S.dtype), s);
            return;
        }
        p.load(a.X.ptr, type(a.X.dtype), row * a.X.ld + i, n);
        if (a.add.ptr) q.load(a.add.ptr, type(a.add.dtype), row * a.add.ld + i, n);
        p.values(type(a.X.dtype), s);
        if (a.add.ptr) {
            float t[8];
            q.values(type(a.add.dtype), t);
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] += t[k];
        }
        if (a.S.ptr) round_to(type(a.S.dtype), s);
    };
    auto each = [&](auto fn, bool again) {  // fn(values, their first, gain), from registers where they were kept
        if (KEPT > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k)
                if (first + k * kStep < whole) fn(x[k], first + k * kStep, gain[k]);
        } else {
            for (int i = first; i < whole; i += kStep) {
                load(i, x[0], again && a.S.ptr);
                if (a.gain.ptr) gain[0].load(a.gain.ptr, type(a.gain.dtype), i, min(max(d - i, 0), 8));
                fn(x[0], i, gain[0]);
            }
        }
    };
    if (KEPT > 0) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) load(first + k * kStep, x[k], false);
        if (a.gain.ptr) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) gain[k].load(a.gain.ptr, type(a.gain.dtype), first + k * kStep, min(max(d - first - k * kStep, 0), 8));
        }
    }
    double sum[kApart ? 4 : 1] = {};
    each([&](float (&s)[8], int i, const Raw8 &) {
        double &part = sum[kApart ? (i - first) / kStep : 0];
#pragma unroll
        for (int k = 0; k < 8; ++k) part = fma((double)s[k], (double)s[k], part);
        if (a.S.ptr && i < d) store_some<8>(a.S.ptr, type(a.S.dtype), row * a.S.ld + i, min(d - i, 8), s);
    }, false);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if constexpr (kApart) {
        const double part = wave_sums_f64(sum);
        if (lane % 16 == 0) sums[(lane >> 5 | (lane >> 4 & 1) << 1) * 4 + wave] = part;
    } else {
        const double part = wave_sum_f64(sum[0]);
        if (lane == 0) sums[wave] = part;
    }
    __syncthreads();
    const double q = total<kApart ? 16 : kWaves>(sums);
    bool bad = !(q < __builtin_huge_val());
    const float r = bad ? (q != q ? __builtin_nanf("") : 0.f) : one_over_root(q * per_value + a.eps);
    auto normed = [&](float (&s)[8], const Raw8 &g) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] *= r;
        if (a.gain.ptr) {
            float t[8];
            g.values(type(a.gain.dtype), t);
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] *= t[k];
        }
    };
    if (!CODED) {
        if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, CMPQ_STATUS_NONFINITE);
        each([&](float (&s)[8], int i, const Raw8 &g) {
            normed(s, g);
            if (i < d) store_some<8>(a.Y.ptr, type(a.Y.dtype), row * a.Y.ld + i, min(d - i, 8), s);
        }, true);
        return;
    }
    Largest largest;
    each([&](float (&s)[8], int, const Raw8 &g) {
        normed(s, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) largest.add(s[k]);
    }, true);
    if (__ballot(largest.bad())) {
        bad = true;
        largest.bits = 0;
        each([&](float (&s)[8], int, const Raw8 &g) {
            if (KEPT == 0) normed(s, g);
#pragma unroll
            for (int k = 0; k < 8; ++k) largest.add_finite(s[k]);
        }, true);
    }
    if (bad && a.status) atomicOr(a.status, CMPQ_STATUS_NONFINITE);
    const float scale = code_scale(block_max(largest.most(), most)), inv = 1.f / scale;
    if (threadIdx.x == 0) a.scale[row] = scale;
    each([&](float (&s)[8], int i, const Raw8 &g) {
        if (KEPT == 0) normed(s, g);
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = bad ? no_nan(s[4 * h + k]) : s[4 * h + k];
            w[h] = low_bytes(code_byte<0>(v[0], inv), code_byte<0>(v[1], inv), code_byte<0>(v[2], inv), code_byte<0>(v[3], inv));
        }
        *reinterpret_cast<uint2 *>(codes + i / kDepth * kPiece + i % kDepth / 16 * 256 + i % 16) = make_uint2(w[0], w[1]);
    }, true);
}

template <int THREADS, int KEPT, bool CODED, int TYPE>
void run(const cmpq_norm_job &a, hipStream_t st) {
    for (int64_t at = 0; at < a.m; at += kRowsOfLaunch) {
        cmpq_norm_job part = a;
        part.m = a.m - at < kRowsOfLaunch ? a.m - at : kRowsOfLaunch;
        for (cmpq_rows *r : {&part.X, &part.add, &part.S, &part.Y})
            if (r->ptr) r->ptr = static_cast<char *>(r->ptr) + at * r->ld * (int64_t)dtype_bytes(r->dtype);
        if (CODED) part.codes += at / kRows * pieces_deep(a.d) * kPiece, part.scale += at;
        const int64_t rows = CODED ? cdiv(part.m, kRows) * kRows : part.m;
        rms_norm_kernel<THREADS, KEPT, CODED, TYPE><<<dim3((unsigned)rows), THREADS, 0, st>>>(part, 1.0 / (double)a.d);
    }
}

// Sixteen wavefronts a row where it is longer than four of them hold in two steps: us with 16 and 4, 1 row of 8192 with its sum
// 3.3 and 4.7, 4096 rows 40.5 and 41.5.  Rows in 8 bits, where there are many, are better off with four, three or four
// steps each, since more of a unit's rows are then at different stages: rows of 5120 (of 8192 with their sum) with 16 and 4, 256 rows 4.44
// and 4.90 (5.51 and 6.45), 320 5.46 and 5.01 (7.26 and 7.10), 512 5.77 and 5.20 (7.72 and 7.83), 576 7.40 and 5.74 (10.1 and 9.3), 1024 9.1 and 6.8
// (14.7 and 14.0), 4096 of 5120 32.3 and 29.
template <bool CODED, int TYPE>
void launch_norm(const cmpq_norm_job &a, hipStream_t st) {
    constexpr int64_t kMany = 512;
    if (a.d <= 2048) run<256, 1, CODED, TYPE>(a, st);
    else if (a.d <= 4096) run<256, 2, CODED, TYPE>(a, st);
    else if (CODED && a.m >= kMany && a.d <= 6144) run<256, CODED ? 3 : 1, CODED, TYPE>(a, st);
    else if (CODED && a.m >= kMany && a.d <= 8192) run<256, CODED ? 4 : 1, CODED, TYPE>(a, st);
    else if (a.d <= 8192) run<1024, 1, CODED, TYPE>(a, st);
    else if (a.d <= 16384) run<1024, 2, CODED, TYPE>(a, st);
    else if (a.d <= 32768) run<1024, 4, CODED, TYPE>(a, st);
    else run<1024, 0, CODED, TYPE>(a, st);
}

}  // namespace

int cmpq_check_rms_norm(const cmpq_norm_job *j) {
    if (!j || j->m < 0 || j->d < 1 || !(j->eps >= 0x1p-126 && j->eps < __builtin_huge_val())) return CMPQ_EINVAL;
    const cmpq_rows all[] = {j->X, j->add, j->gain, j->S, j->Y};
    for (const cmpq_rows &a : all)
        if (a.ptr && !serving_dtype(a.dtype)) return CMPQ_EINVAL;
    if (j->m == 0) return CMPQ_OK;
    if (!j->Y.ptr == !j->codes || (j->codes && (!j->scale || reinterpret_cast<uintptr_t>(j->codes) % 16))) return CMPQ_EINVAL;
    if (!j->X.ptr) return CMPQ_EINVAL;
    if (j->m >= (1 << 24) || j->d > kMostDepth) return CMPQ_ESHAPE;
    const cmpq_rows rows[] = {j->X, j->add, j->S, j->Y};
    for (const cmpq_rows &a : rows)
        if (a.ptr && a.ld < j->d) return CMPQ_ESHAPE;
    return CMPQ_OK;
}

extern "C" int cmpq_rms_norm(const cmpq_norm_job *j, void *stream) {
    if (int rc = cmpq_check_rms_norm(j)) return rc;
    if (j->m == 0) return CMPQ_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const cmpq_rows all[] = {j->X, j->add, j->gain, j->S, j->Y};
    int type = j->X.dtype;
    for (const cmpq_rows &a : all)
        if (a.ptr && a.dtype != j->X.dtype) type = kAny;
    if (j->codes) {
        if (type == CMPQ_F16) launch_norm<true, CMPQ_F16>(*j, st);
        else if (type == CMPQ_BF16) launch_norm<true, CMPQ_BF16>(*j, st);
        else launch_norm<true, kAny>(*j, st);
    } else {
        if (type == CMPQ_F16) launch_norm<false, CMPQ_F16>(*j, st);
        else if (type == CMPQ_BF16) launch_norm<false, CMPQ_BF16>(*j, st);
        else launch_norm<false, kAny>(*j, st);
    }
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
