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

// Workgroups in the order in which they are handed to the eight dies, so that each die gets a run of them.
__device__ __forceinline__ int64_t die_order(int64_t x, int64_t n) {
    const int64_t each = n / 8, more = n % 8, die = x % 8;
    return die * each + min(die, more) + x / 8;
}

// Sixteen inputs of a row as they lie in memory; `valid` of them are there, the others read 0.
template <typename T>
struct Sixteen {
    typedef T V __attribute__((ext_vector_type(16)));
    V v;
    __device__ __forceinline__ void load(const T *p, int64_t valid) {
        typedef V Any __attribute__((aligned(sizeof(T))));
        if (valid >= 16) {
            v = *reinterpret_cast<const Any *>(p);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = i < valid ? p[i] : (T)0.f;
        }
    }
};

// One workgroup a row: its largest magnitude, then its codes, 16 inputs a lane and step.  Rows of up to KEPT * 4096
// inputs stay in registers between the two, longer ones are read again.  The rows of a piece write 16 bytes each
// of the same lines, so consecutive rows go to one die, whose cache puts the lines together.
template <typename T, int KEPT>
__global__ __launch_bounds__(256) void code_rows_kernel(const T *__restrict__ X, int64_t n, int64_t d, int64_t ld,
                                                        int8_t *__restrict__ codes, float *__restrict__ scale,
                                                        int32_t *__restrict__ status) {
    __shared__ float scratch[4];
    const int64_t row = die_order(blockIdx.x, gridDim.x), deep = pieces_deep(d);
    uint8_t *out = reinterpret_cast<uint8_t *>(codes) + row / kRows * deep * kPiece + row % kRows * 16;
    const int groups = (int)deep * 4;
    if (row >= n) {  // rows that fill up the last piece
        for (int c = threadIdx.x; c < groups; c += 256)
            *reinterpret_cast<uint4 *>(out + c / 4 * kPiece + c % 4 * 256) = make_uint4(0, 0, 0, 0);
        return;
    }
    const T *x = X + row * ld;
    float most = 0.f;
    bool bad = false;
    Sixteen<T> kept[KEPT > 0 ? KEPT : 1];
    auto look = [&](const Sixteen<T> &s) {
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, finite_abs((float)s.v[i], bad));
    };
    auto code = [&](const Sixteen<T> &s, int c, float inv) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i] |= (uint32_t)(code_of((float)s.v[4 * i + j], inv) & 255) << (8 * j);
        }
        *reinterpret_cast<uint4 *>(out + c / 4 * kPiece + c % 4 * 256) = make_uint4(w[0], w[1], w[2], w[3]);
    };
    if (KEPT > 0) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            const int c = threadIdx.x + k * 256;
            kept[k].load(x + c * 16, c < groups ? d - c * 16 : 0);
        }
#pragma unroll
        for (int k = 0; k < KEPT; ++k) look(kept[k]);
    } else {
        for (int c = threadIdx.x; c < groups; c += 256) {
            kept[0].load(x + c * 16, d - c * 16);
            look(kept[0]);
        }
    }
    most = block_max(most, scratch);
    const float s = code_scale(most), inv = 1.f / s;
    if (threadIdx.x == 0) scale[row] = s;
    if (bad && status) atomicOr(status, CMPQ_STATUS_NONFINITE);
    if (KEPT > 0) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k)
            if (threadIdx.x + k * 256 < groups) code(kept[k], threadIdx.x + k * 256, inv);
    } else {
        for (int c = threadIdx.x; c < groups; c += 256) {
            kept[0].load(x + c * 16, d - c * 16);
            code(kept[0], c, inv);
        }
    }
}

template <typename T>
void launch_code_rows(const void *X, int64_t n, int64_t d, int64_t ld, int64_t rows, int8_t *codes, float *scale,
                      int32_t *status, hipStream_t st) {
    const dim3 grid((unsigned)rows);
    const T *x = static_cast<const T *>(X);
    if (d <= 4096) code_rows_kernel<T, 1><<<grid, 256, 0, st>>>(x, n, d, ld, codes, scale, status);
    else if (d <= 8192) code_rows_kernel<T, 2><<<grid, 256, 0, st>>>(x, n, d, ld, codes, scale, status);
    else if (d <= 16384) code_rows_kernel<T, 4><<<grid, 256, 0, st>>>(x, n, d, ld, codes, scale, status);
    else code_rows_kernel<T, 0><<<grid, 256, 0, st>>>(x, n, d, ld, codes, scale, status);
}

// `rows` of them, those from n on zeros.
int launch_code_rows_of(const void *X, int dtype, int64_t n, int64_t d, int64_t ld, int64_t rows, int8_t *codes,
                     float *scale, int32_t *status, hipStream_t st) {
    if (dtype == CMPQ_F16) launch_code_rows<_Float16>(X, n, d, ld, rows, codes, scale, status, st);
    else if (dtype == CMPQ_BF16) launch_code_rows<__bf16>(X, n, d, ld, rows, codes, scale, status, st);
    else launch_code_rows<float>(X, n, d, ld, rows, codes, scale, status, st);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

struct Scaled {
    const float *sx, *sw;
    void *Y;
    int64_t m, d_out, ldy;
    bool aligned;  // four outputs next to each other may be written at once
};

// The smaller scale first: a sum that is not 0 times a scale of at least 2^-126 neither vanishes nor, where the
// result is in range, overflows on the way.
__device__ __forceinline__ float scaled(int sum, float sx, float sw) {
    return (float)sum * fminf(sx, sw) * fmaxf(sx, sw);
}

// Four outputs next to each other, o .. o + 3, of token t.
template <typename T>
__device__ __forceinline__ void put4(const Scaled &y, int64_t t, int64_t o, const Int4 &acc) {
    if (t >= y.m || o >= y.d_out) return;
    const float sx = y.sx[t];
    T *p = static_cast<T *>(y.Y) + t * y.ldy + o;
    if (o + 4 <= y.d_out && y.aligned) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        const float4 sw = *reinterpret_cast<const float4 *>(y.sw + o);
        *reinterpret_cast<T4 *>(p) = T4{(T)scaled(acc[0], sx, sw.x), (T)scaled(acc[1], sx, sw.y),
                                        (T)scaled(acc[2], sx, sw.z), (T)scaled(acc[3], sx, sw.w)};
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (o + r < y.d_out) p[r] = (T)scaled(acc[r], sx, y.sw[o + r]);
    }
}

__device__ __forceinline__ Int4 multiply(const Int4 &w, const Int4 &x, const Int4 &acc) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
}

// Few outputs or tokens: a workgroup has OP x TP pieces of 16 outputs by 16 tokens, its wavefronts share the depth and
// add up through LDS.  Operands come straight from memory, kAhead steps of 64 inputs at once.
template <typename T, int OP, int TP, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void shared_depth_kernel(const uint8_t *__restrict__ W,
                                                                  const uint8_t *__restrict__ X, int deep, Scaled y) {
    constexpr int kAhead = OP + TP <= 3 ? 4 : 2;
    __shared__ Int4 red[WAVES][OP * TP][64];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int64_t o0 = (int64_t)blockIdx.x * OP, t0 = (int64_t)blockIdx.y * TP;
    const int64_t last_o = (y.d_out - 1) / kRows, last_t = (y.m - 1) / kRows;
    const uint8_t *w[OP], *x[TP];
#pragma unroll
    for (int i = 0; i < OP; ++i) w[i] = W + min(o0 + i, last_o) * deep * kPiece + lane * 16;
#pragma unroll
    for (int i = 0; i < TP; ++i) x[i] = X + min(t0 + i, last_t) * deep * kPiece + lane * 16;
    Int4 acc[OP][TP] = {};
    const int k0 = (int)((int64_t)deep * wave / WAVES), k1 = (int)((int64_t)deep * (wave + 1) / WAVES);
    for (int k = k0; k < k1; k += kAhead) {
        Int4 a[kAhead][OP], b[kAhead][TP];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = min(k + u, k1 - 1) * kPiece;
#pragma unroll
            for (int i = 0; i < OP; ++i) a[u][i] = *reinterpret_cast<const Int4 *>(w[i] + at);
#pragma unroll
            for (int i = 0; i < TP; ++i) b[u][i] = *reinterpret_cast<const Int4 *>(x[i] + at);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k + u >= k1) break;
#pragma unroll
            for (int i = 0; i < OP; ++i)
#pragma unroll
                for (int j = 0; j < TP; ++j) acc[i][j] = multiply(a[u][i], b[u][j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < OP; ++i)
#pragma unroll
        for (int j = 0; j < TP; ++j) red[wave][i * TP + j][lane] = acc[i][j];
    __syncthreads();
    for (int q = wave; q < OP * TP; q += WAVES) {
        Int4 sum = red[0][q][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += red[v][q][lane];
        put4<T>(y, (t0 + q % TP) * kRows + (lane & 15), (o0 + q / TP) * kRows + (lane >> 4) * 4, sum);
    }
}

__device__ __forceinline__ void load_lds16(const uint8_t *src, uint8_t *dst) {
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) uint32_t *>(reinterpret_cast<uintptr_t>(src)),
                                     reinterpret_cast<__attribute__((address_space(3))) uint32_t *>((uint32_t)reinterpret_cast<uintptr_t>(dst)), 16, 0, 0);
}

// Many tokens: 256 outputs by 256 tokens a workgroup of 8 wavefronts, 128 by 64 a wavefront.  Pieces reach LDS by direct
// loads in the order in which they are read (no conflicts); a step of 64 inputs is one buffer of 32 KB, and
// kBuffers - 1 steps are on their way while one is multiplied.
constexpr int kTile = 16, kStepBytes = 2 * kTile * kPiece, kBuffers = 4, kBand = 4;

template <typename T>
__global__ __launch_bounds__(512, 2) void tile_kernel(const uint8_t *__restrict__ W, const uint8_t *__restrict__ X,
                                                      int deep, int o_tiles, int t_tiles, Scaled y) {
    __shared__ __align__(16) uint8_t smem[kBuffers * kStepBytes];
    const int lane = threadIdx.x & 63, wave = wave_index();
    // bands of kBand token tiles, all output tiles of a band one after the other
    const int64_t n = die_order(blockIdx.x, (int64_t)o_tiles * t_tiles);
    const int band = (int)(n / ((int64_t)kBand * o_tiles)), in_band = (int)(n - (int64_t)band * kBand * o_tiles);
    const int wide = min(kBand, t_tiles - band * kBand);
    const int64_t o0 = (int64_t)(in_band / wide) * kTile, t0 = (int64_t)(band * kBand + in_band % wide) * kTile;
    const int64_t last_o = (y.d_out - 1) / kRows, last_t = (y.m - 1) / kRows;
    // wavefronts 0..3 bring 4 pieces of W each, the others of X
    const uint8_t *src[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = 4 * (wave & 3) + q;
        src[q] = (wave < 4 ? W + min(o0 + k, last_o) * deep * kPiece : X + min(t0 + k, last_t) * deep * kPiece) + lane * 16;
    }
    uint8_t *dst = smem + wave * 4 * kPiece;
    auto load = [&](int step) {  // past the last step: that one again, which nothing reads
        const int64_t at = (int64_t)min(step, deep - 1) * kPiece;
        uint8_t *to = dst + (step % kBuffers) * kStepBytes;
#pragma unroll
        for (int q = 0; q < 4; ++q) load_lds16(src[q] + at, to + q * kPiece);
    };
    const int wo = (wave & 1) * 8, wt = (wave >> 1) * 4;
    Int4 acc[8][4] = {};
#pragma unroll
    for (int u = 0; u < kBuffers - 1; ++u) load(u);
    for (int step = 0; step < deep; ++step) {
        // This wavefront's 4 loads of the oldest step have landed (two later steps, 8 loads, are under way) and its LDS
        // reads of the step before have returned.  After the barrier both hold for every wavefront.
        static_assert(kBuffers == 4, "the count of loads still under way");
        asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load(step + kBuffers - 1);
        const uint8_t *buf = smem + (step % kBuffers) * kStepBytes + lane * 16;
        Int4 a[8], b[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) b[q] = *reinterpret_cast<const Int4 *>(buf + (kTile + wt + q) * kPiece);
#pragma unroll
        for (int q = 0; q < 8; ++q) a[q] = *reinterpret_cast<const Int4 *>(buf + (wo + q) * kPiece);
#pragma unroll
        for (int p = 0; p < 8; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[p][q] = multiply(a[p], b[q], acc[p][q]);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads that nothing reads end before the LDS does
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int p = 0; p < 8; ++p)
            put4<T>(y, (t0 + wt + q) * kRows + (lane & 15), (o0 + wo + p) * kRows + (lane >> 4) * 4, acc[p][q]);
}

template <typename T, int OP, int TP, int WAVES>
void launch_shared(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, hipStream_t st) {
    const dim3 grid((unsigned)cdiv(y.d_out, OP * kRows), (unsigned)cdiv(y.m, TP * kRows));
    shared_depth_kernel<T, OP, TP, WAVES><<<grid, WAVES * 64, 0, st>>>(W, X, deep, y);
}

template <typename T>
int launch_product(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, hipStream_t st) {
    const int o_tiles = (int)cdiv(y.d_out, kTile * kRows), t_tiles = (int)cdiv(y.m, kTile * kRows);
    if (y.m <= 16) {
        if (cdiv(y.d_out, 32) >= 512) launch_shared<T, 2, 1, 8>(W, X, deep, y, st);
        else launch_shared<T, 1, 1, 16>(W, X, deep, y, st);
    } else if (y.m <= 32) {
        launch_shared<T, 2, 2, 8>(W, X, deep, y, st);
    } else if ((int64_t)o_tiles * t_tiles < 200 && cdiv(y.m, 64) < 65536) {
        launch_shared<T, 4, 4, 4>(W, X, deep, y, st);
    } else {
        if ((int64_t)o_tiles * t_tiles > INT32_MAX) return CMPQ_ESHAPE;
        tile_kernel<T><<<dim3((unsigned)(o_tiles * t_tiles)), 512, 0, st>>>(W, X, deep, o_tiles, t_tiles, y);
    }
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
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
    return launch_code_rows_of(W, dtype, d_out, d_in, ldw, cdiv(d_out, kRows) * kRows, codes, scale, status,
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
    if (int rc = launch_code_rows_of(X, dtype, m, d_in, ldx, m, w.codes, w.scale, status, st)) return rc;
    const size_t four = 4 * dtype_bytes(y_dtype);
    const Scaled y = {w.scale, scale, Y, m, d_out, ldy,
                      ldy % 4 == 0 && reinterpret_cast<uintptr_t>(Y) % four == 0 && reinterpret_cast<uintptr_t>(scale) % 16 == 0};
    const uint8_t *cw = reinterpret_cast<const uint8_t *>(codes), *cx = reinterpret_cast<const uint8_t *>(w.codes);
    const int deep = (int)pieces_deep(d_in);
    if (y_dtype == CMPQ_F16) return launch_product<_Float16>(cw, cx, deep, y, st);
    if (y_dtype == CMPQ_BF16) return launch_product<__bf16>(cw, cx, deep, y, st);
    return launch_product<float>(cw, cx, deep, y, st);
}
