// Products in 8-bit integers: codes with a scale per row of either operand, exact sums, one multiplication by each
// scale at the end.  Both operands lie in pieces of 16 rows by 64 inputs (1 KB), byte [g][r][j] of a piece being row r,
// input 16 g + j: what lane 16 g + r of a wavefront hands the 16x16x64 matrix instruction is 16 bytes in order, and
// a wavefront's load is 1 KB in order, from memory and from LDS alike.
#include "serving.h"

namespace {

typedef int32_t Int4 __attribute__((ext_vector_type(4)));

constexpr int kRows = 16, kDepth = 64, kPiece = kRows * kDepth;  // a piece
constexpr int64_t kMostDepth = 131072;                            // 127 * 127 * d_in < 2^31

__host__ __device__ inline int64_t pieces_deep(int64_t d) { return (d + 127) / 128 * 2; }

// One workgroup a row: its largest magnitude, then its codes, 16 inputs a lane.
template <typename T>
__global__ __launch_bounds__(256) void code_rows_kernel(const T *__restrict__ X, int64_t n, int64_t d, int64_t ld,
                                                        int8_t *__restrict__ codes, float *__restrict__ scale,
                                                        int32_t *__restrict__ status) {
    __shared__ float scratch[4];
    const int64_t row = blockIdx.x, deep = pieces_deep(d);
    uint8_t *out = reinterpret_cast<uint8_t *>(codes) + row / kRows * deep * kPiece + row % kRows * 16;
    const int64_t groups = deep * 4;
    if (row >= n) {  // rows that fill up the last piece
        for (int64_t c = threadIdx.x; c < groups; c += 256)
            *reinterpret_cast<uint4 *>(out + c / 4 * kPiece + c % 4 * 256) = make_uint4(0, 0, 0, 0);
        return;
    }
    const T *x = X + row * ld;
    float most = 0.f;
    bool bad = false;
    for (int64_t c = threadIdx.x; c < groups; c += 256) {
        float v[16];
        load_f32<T, 16>(x + c * 16, (int)min((int64_t)16, max((int64_t)0, d - c * 16)), v);
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, finite_abs(v[i], bad));
    }
    most = block_max(most, scratch);
    const float s = code_scale(most), inv = 1.f / s;
    if (threadIdx.x == 0) scale[row] = s;
    if (bad && status) atomicOr(status, CMPQ_STATUS_NONFINITE);
    for (int64_t c = threadIdx.x; c < groups; c += 256) {
        float v[16];
        load_f32<T, 16>(x + c * 16, (int)min((int64_t)16, max((int64_t)0, d - c * 16)), v);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i] |= (uint32_t)(code_of(v[4 * i + j], inv) & 255) << (8 * j);
        }
        *reinterpret_cast<uint4 *>(out + c / 4 * kPiece + c % 4 * 256) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// `rows` of them, those from n on zeros.
int launch_code_rows(const void *X, int dtype, int64_t n, int64_t d, int64_t ld, int64_t rows, int8_t *codes,
                     float *scale, int32_t *status, hipStream_t st) {
    const dim3 grid((unsigned)rows);
    if (dtype == CMPQ_F16)
        code_rows_kernel<_Float16><<<grid, 256, 0, st>>>(static_cast<const _Float16 *>(X), n, d, ld, codes, scale, status);
    else if (dtype == CMPQ_BF16)
        code_rows_kernel<__bf16><<<grid, 256, 0, st>>>(static_cast<const __bf16 *>(X), n, d, ld, codes, scale, status);
    else
        code_rows_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float *>(X), n, d, ld, codes, scale, status);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

struct Scaled {
    const float *sx, *sw;
    void *Y;
    int64_t m, d_out, ldy;
    int dtype;
};

// The smaller scale first: a sum that is not 0 times a scale of at least 2^-126 neither vanishes nor, where the
// result is in range, overflows on the way.
__device__ __forceinline__ float scaled(int sum, float sx, float sw) {
    return (float)sum * fminf(sx, sw) * fmaxf(sx, sw);
}

// Four outputs next to each other of token t.
__device__ __forceinline__ void put4(const Scaled &y, int64_t t, int64_t o, const Int4 &acc) {
    if (t >= y.m) return;
    const float sx = y.sx[t];
    with_dtype(y.dtype, [&](auto like) {
        using T = decltype(like);
        T *p = static_cast<T *>(y.Y) + t * y.ldy + o;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (o + r < y.d_out) p[r] = (T)scaled(acc[r], sx, y.sw[o + r]);
    });
}

// 128 outputs by 128 tokens a workgroup, 64 by 64 a wavefront, operands straight from memory.
__global__ __launch_bounds__(256) void product_kernel(const uint8_t *__restrict__ W, const uint8_t *__restrict__ X,
                                                      int64_t deep, Scaled y) {
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int64_t o0 = (int64_t)blockIdx.x * 128 + (wave & 1) * 64, t0 = (int64_t)blockIdx.y * 128 + (wave >> 1) * 64;
    const int64_t last_o = (y.d_out - 1) / kRows, last_t = (y.m - 1) / kRows;
    const uint8_t *w[4], *x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = W + min(o0 / kRows + i, last_o) * deep * kPiece + lane * 16;
        x[i] = X + min(t0 / kRows + i, last_t) * deep * kPiece + lane * 16;
    }
    Int4 acc[4][4] = {};
    for (int64_t k = 0; k < deep; ++k) {
        Int4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = *reinterpret_cast<const Int4 *>(w[i] + k * kPiece);
            b[i] = *reinterpret_cast<const Int4 *>(x[i] + k * kPiece);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) put4(y, t0 + j * 16 + (lane & 15), o0 + i * 16 + (lane >> 4) * 4, acc[i][j]);
}

struct Work {
    int8_t *codes;
    float *scale;
    size_t bytes;
};
Work carve(void *ws, int64_t m, int64_t d_in) {
    WsCarver c(ws);
    Work w;
    w.codes = c.take<int8_t>((size_t)(cdiv(m, kRows) * pieces_deep(d_in) * kPiece));
    w.scale = c.take<float>((size_t)m);
    w.bytes = c.need();
    return w;
}

bool sizes_fit(int64_t d_in, int64_t d_out) { return d_in <= kMostDepth && d_out < (1 << 24); }

}  // namespace

size_t cmpq_ws_int8_product(int64_t d_in, int64_t m) { return carve(nullptr, m > 0 ? m : 1, d_in).bytes; }

extern "C" size_t cmpq_int8_weight_bytes(int64_t d_out, int64_t d_in) {
    if (d_out < 0 || d_in < 0 || !sizes_fit(d_in, d_out)) return 0;
    return (size_t)(cdiv(d_out, kRows) * pieces_deep(d_in) * kPiece);
}

extern "C" int cmpq_int8_prepare(const void *W, int dtype, int64_t d_out, int64_t d_in, int64_t ldw, int8_t *codes,
                                 float *scale, int32_t *status, void *stream) {
    if (d_out < 0 || d_in < 0 || !serving_dtype(dtype)) return CMPQ_EINVAL;
    if (d_out == 0 || d_in == 0) return CMPQ_OK;
    if (!W || !codes || !scale || reinterpret_cast<uintptr_t>(codes) % 16) return CMPQ_EINVAL;
    if (ldw < d_in || !sizes_fit(d_in, d_out)) return CMPQ_ESHAPE;
    return launch_code_rows(W, dtype, d_out, d_in, ldw, cdiv(d_out, kRows) * kRows, codes, scale, status,
                            static_cast<hipStream_t>(stream));
}

extern "C" int cmpq_int8_product(const void *X, int dtype, int64_t m, int64_t d_in, int64_t ldx, const int8_t *codes,
                                 const float *scale, int64_t d_out, void *Y, int y_dtype, int64_t ldy, void *ws,
                                 size_t ws_bytes, int32_t *status, void *stream) {
    if (m < 0 || d_in < 1 || d_out < 0 || !serving_dtype(dtype) || !serving_dtype(y_dtype)) return CMPQ_EINVAL;
    if (m == 0 || d_out == 0) return CMPQ_OK;
    if (!X || !codes || !scale || !Y || reinterpret_cast<uintptr_t>(codes) % 16) return CMPQ_EINVAL;
    if (ldx < d_in || ldy < d_out || m >= (1 << 24) || !sizes_fit(d_in, d_out)) return CMPQ_ESHAPE;
    const Work w = carve(ws, m, d_in);
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < w.bytes) return CMPQ_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int rc = launch_code_rows(X, dtype, m, d_in, ldx, m, w.codes, w.scale, status, st)) return rc;
    const Scaled y = {w.scale, scale, Y, m, d_out, ldy, y_dtype};
    const dim3 grid((unsigned)cdiv(d_out, 128), (unsigned)cdiv(m, 128));
    if (grid.y > 65535) return CMPQ_ESHAPE;
    product_kernel<<<grid, 256, 0, st>>>(reinterpret_cast<const uint8_t *>(codes),
                                         reinterpret_cast<const uint8_t *>(w.codes), pieces_deep(d_in), y);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
