// What the calls of 8-bit serving share: element types, the one rule of all 8-bit codes, the position rotation and
// the checks of their arguments.
#pragma once

#include "common.h"

constexpr float kSmallestScale = 0x1p-126f;  // keeps 1 / scale finite; also the scale of zeros

template <typename T>
__device__ __forceinline__ float as_f32(T v) {
    return (float)v;
}

// fn(T()) for the element type that `dtype` names; the host has checked that it names one.
template <typename F>
__device__ __forceinline__ void with_dtype(int dtype, F fn) {
    if (dtype == CMPQ_F16) fn(_Float16());
    else if (dtype == CMPQ_BF16) fn(__bf16());
    else fn(float());
}

static inline bool serving_dtype(int dtype) { return dtype == CMPQ_F16 || dtype == CMPQ_BF16 || dtype == CMPQ_F32; }
static inline size_t dtype_bytes(int dtype) { return dtype == CMPQ_F32 ? 4 : 2; }

// N elements next to each other in 32 bits, at any alignment of their type.
template <typename T, int N>
__device__ __forceinline__ void load_f32(const T *p, float (&x)[N]) {
    typedef T V __attribute__((ext_vector_type(N)));
    typedef V Any __attribute__((aligned(sizeof(T))));
    const V v = *reinterpret_cast<const Any *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}

// Largest magnitude of values, and whether all were finite: magnitudes are ordered as their bits are, infinity and NaN
// above the rest.  Where one was not finite (bad()), they are looked over again without those.
struct Largest {
    uint32_t bits = 0;
    static constexpr uint32_t kInfinity = 0x7f800000u;
    __device__ __forceinline__ void add(float x) { bits = max(bits, __float_as_uint(x) & 0x7fffffffu); }
    __device__ __forceinline__ void add_finite(float x) {
        const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
        bits = a < kInfinity ? max(bits, a) : bits;
    }
    __device__ __forceinline__ bool bad() const { return bits >= kInfinity; }
    __device__ __forceinline__ float most() const { return __uint_as_float(bits); }
};

__device__ __forceinline__ float code_scale(float most) { return fmaxf(most / 127.f, kSmallestScale); }

// x * inv within -127..127, rounded to even, in the low byte (two's complement; OFFSET more): adding 3 * 2^22 rounds and
// leaves the number there.  x is no NaN.
template <int OFFSET>
__device__ __forceinline__ uint32_t code_byte(float x, float inv) {
    return __float_as_uint(__builtin_amdgcn_fmed3f(x * inv, -127.f, 127.f) + (float)(12582912 + OFFSET));
}
// The low bytes of four words next to each other.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
}
__device__ __forceinline__ float no_nan(float x) { return x == x ? x : 0.f; }

// The value of the lane N further on in a row of 16, around its end.
template <int N>
__device__ __forceinline__ uint32_t row_turn(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xF, 0xF, true);
}
// Largest of a row of 16 lanes, in all of them.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    v = max(v, row_turn<8>(v));
    v = max(v, row_turn<4>(v));
    v = max(v, row_turn<2>(v));
    return max(v, row_turn<1>(v));
}

// Largest of non-negative values over the workgroup of up to 16 wavefronts, in every lane.  `scratch`: one float a wavefront.
// Has a barrier.  Values are ordered as their bits are.  Row swaps and the DPP path: exchanges through LDS and a loop over the
// wavefronts took 16 of them a microsecond longer.
__device__ __forceinline__ float block_max(float value, float *scratch) {
    uint32_t v = __float_as_uint(value);
    const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(halves[0], halves[1]);
    const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = row_max(max(rows[0], rows[1]));
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = __uint_as_float(v);
    __syncthreads();
    const int w = threadIdx.x & 15;
    return __uint_as_float(row_max(w < (int)(blockDim.x >> 6) ? __float_as_uint(scratch[w]) : 0));
}

// The same of four rows that lie in turn from lane to lane of 16 wavefronts.  `scratch`: 64 floats.
__device__ __forceinline__ float four_rows_max(float value, float *scratch) {
    const auto join = [](uint32_t v) {
        v = max(v, row_turn<8>(v));
        v = max(v, row_turn<4>(v));
        const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(halves[0], halves[1]);
        const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return max(rows[0], rows[1]);
    };
    const uint32_t v = join(__float_as_uint(value));
    const int lane = threadIdx.x & 63;
    if (lane < 4) scratch[(threadIdx.x >> 6) * 4 + lane] = __uint_as_float(v);
    __syncthreads();
    return __uint_as_float(join(__float_as_uint(scratch[lane])));  // a wavefront's four, then the next one's
}

// The two results of the turn by position.  Products and sums are rounded one by one, as the header says.
__device__ __forceinline__ float turned_first(float a, float b, float c, float s) {
#pragma clang fp contract(off)
    const float ac = a * c, bs = b * s;
    return ac - bs;
}
__device__ __forceinline__ float turned_second(float a, float b, float c, float s) {
#pragma clang fp contract(off)
    const float bc = b * c, as = a * s;
    return bc + as;
}

// Dim `d` of a head at `p` turned for the row `at` of the tables (null: not turned).
template <typename T>
__device__ __forceinline__ float turned(const T *p, int d, const cmpq_rotation &rot, int64_t at) {
    const float x = (float)p[d];
    if (!rot.cos || d >= rot.dims) return x;
    const int half = rot.dims >> 1;
    const int j = rot.interleaved ? d >> 1 : (d < half ? d : d - half);
    const bool second = rot.interleaved ? d & 1 : d >= half;
    const int other = rot.interleaved ? d ^ 1 : (second ? d - half : d + half);
    const float y = (float)p[other], c = rot.cos[at * half + j], s = rot.sin[at * half + j];
    return second ? turned_second(y, x, c, s) : turned_first(x, y, c, s);
}

// Whether the turn's pairs are eight next to each other, like the eight dims they are taken for, or lie within the eight.
__host__ __device__ __forceinline__ bool turns_by_eight(const cmpq_rotation &rot) {
    return !rot.cos || (rot.interleaved ? rot.dims % 8 == 0 : rot.dims % 16 == 0);
}

// Dims d .. d + 7 (d a multiple of 8, all within the head) at `p`, turned by eight for the row of the tables that begins at
// element `row`.
template <typename T>
__device__ __forceinline__ void load_turned(const T *p, int d, const cmpq_rotation &rot, int64_t row, float (&x)[8]) {
    load_f32<T, 8>(p + d, x);
    if (!rot.cos || d >= rot.dims) return;
    const int half = rot.dims >> 1;
    if (rot.interleaved) {
        float cs[4], sn[4];
        load_f32<float, 4>(rot.cos + row + d / 2, cs);
        load_f32<float, 4>(rot.sin + row + d / 2, sn);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float a = x[i], b = x[i + 1];
            x[i] = turned_first(a, b, cs[i / 2], sn[i / 2]);
            x[i + 1] = turned_second(a, b, cs[i / 2], sn[i / 2]);
        }
    } else {
        const bool second = d >= half;
        const int pair = second ? d - half : d;
        const uint32_t flip = second ? 0x80000000u : 0;  // b cos + a sin = b cos - a (-sin), bit for bit
        float y[8], cs[8], sn[8];
        load_f32<T, 8>(p + (second ? pair : d + half), y);
        load_f32<float, 8>(rot.cos + row + pair, cs);
        load_f32<float, 8>(rot.sin + row + pair, sn);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = turned_first(x[i], y[i], cs[i], __uint_as_float(__float_as_uint(sn[i]) ^ flip));
    }
}

static inline int check_rotation(const cmpq_rotation *rot, int head_dim) {
    if (!rot || !rot->cos) return CMPQ_OK;
    if (!rot->sin || rot->positions < 1 || rot->dims < 2 || (rot->dims & 1)) return CMPQ_EINVAL;
    return rot->dims <= head_dim ? CMPQ_OK : CMPQ_ESHAPE;
}

static inline int check_cache(const cmpq_kv_cache &c) {
    if (!c.k_codes || !c.v_codes || !c.k_scale || !c.v_scale || c.n_pages < 0 || c.kv_heads < 1) return CMPQ_EINVAL;
    if (!cmpq_kv_page_bytes(c.head_dim, c.page) || c.kv_heads > 65535 || c.n_pages > INT32_MAX) return CMPQ_ESHAPE;
    if (reinterpret_cast<uintptr_t>(c.k_codes) % 16 || reinterpret_cast<uintptr_t>(c.v_codes) % 16) return CMPQ_EINVAL;
    return CMPQ_OK;
}

// Of 2^32 lanes or more HIP launches what 32 bits hold of the number, as a rule without an error.
static inline bool one_launch(int64_t workgroups, int lanes) { return workgroups <= (int64_t)UINT32_MAX / lanes; }

// For calls that do no row: CMPQ_STATUS_RANGE where a sequence names one all the same.
int cmpq_flag_named_rows(const int32_t *cu, int64_t n_seq, int32_t *status, hipStream_t stream);
