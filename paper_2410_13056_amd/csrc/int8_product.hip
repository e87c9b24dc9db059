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
    __device__ __forceinline__ void look(Largest &l) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) l.add((float)v[i]);
    }
    __device__ __forceinline__ void look_again(Largest &l) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) l.add_finite((float)v[i]);
    }
    // `clean`: none is a NaN.
    __device__ __forceinline__ uint4 codes(float inv, bool clean) const {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = (float)v[4 * i + k];
                if (!clean) x[k] = no_nan(x[k]);
            }
            w[i] = low_bytes(code_byte<0>(x[0], inv), code_byte<0>(x[1], inv), code_byte<0>(x[2], inv), code_byte<0>(x[3], inv));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// One workgroup a row: its largest magnitude, then its codes, 16 inputs a lane and step.  Rows of up to KEPT * 4096
// inputs stay in registers between the two, longer ones are read again.  The rows of a piece write 16 bytes each
// of the same lines, so consecutive rows go to one die, whose cache puts the lines together.  Bound by bytes where rows are
// many: 4096 rows of 8192 in FP16 29 us, 3.5 TB/s (three quarters of a copy's rate; vector instructions 38 %); by a row's latency
// where they are few: 333 rows 4 us.
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
    Largest largest;
    Sixteen<T> kept[KEPT > 0 ? KEPT : 1];
    auto each = [&](auto fn) {  // fn(sixteen inputs, their number), from registers where they were kept
        if (KEPT > 0) {
#pragma unroll
            for (int k = 0; k < KEPT; ++k)
                if ((int)threadIdx.x + k * 256 < groups) fn(kept[k], (int)threadIdx.x + k * 256);
        } else {
            for (int c = threadIdx.x; c < groups; c += 256) {
                kept[0].load(x + c * 16, d - c * 16);
                fn(kept[0], c);
            }
        }
    };
    if (KEPT > 0) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            const int c = threadIdx.x + k * 256;
            kept[k].load(x + c * 16, c < groups ? d - c * 16 : 0);
        }
    }
    each([&](const Sixteen<T> &s, int) { s.look(largest); });
    const bool bad = __ballot(largest.bad()) != 0;
    if (bad) {
        largest.bits = 0;
        each([&](const Sixteen<T> &s, int) { s.look_again(largest); });
        if (status) atomicOr(status, CMPQ_STATUS_NONFINITE);
    }
    const float s = code_scale(block_max(largest.most(), scratch)), inv = 1.f / s;
    if (threadIdx.x == 0) scale[row] = s;
    auto put = [&](const Sixteen<T> &s, int c, bool clean) {
        *reinterpret_cast<uint4 *>(out + c / 4 * kPiece + c % 4 * 256) = s.codes(inv, clean);
    };
    if (bad) each([&](const Sixteen<T> &s, int c) { put(s, c, false); });
    else each([&](const Sixteen<T> &s, int c) { put(s, c, true); });
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

__device__ __forceinline__ float token_scale(const Scaled &y, int64_t t) { return t < y.m ? y.sx[t] : 0.f; }

// Of outputs o .. o + 3.
__device__ __forceinline__ float4 output_scales(const Scaled &y, int64_t o) {
    if (o + 4 <= y.d_out && y.aligned) return *reinterpret_cast<const float4 *>(y.sw + o);
    const auto one = [&](int64_t i) { return i < y.d_out ? y.sw[i] : 0.f; };
    return make_float4(one(o), one(o + 1), one(o + 2), one(o + 3));
}

// Four outputs next to each other, o .. o + 3, of token t.
template <typename T>
__device__ __forceinline__ void put4(const Scaled &y, int64_t t, int64_t o, const Int4 &acc, float sx, const float4 &sw) {
    if (t >= y.m || o >= y.d_out) return;
    T *p = static_cast<T *>(y.Y) + t * y.ldy + o;
    typedef T T4 __attribute__((ext_vector_type(4)));
    const T4 v = {(T)scaled(acc[0], sx, sw.x), (T)scaled(acc[1], sx, sw.y), (T)scaled(acc[2], sx, sw.z), (T)scaled(acc[3], sx, sw.w)};
    if (o + 4 <= y.d_out && y.aligned) {
        *reinterpret_cast<T4 *>(p) = v;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (o + r < y.d_out) p[r] = v[r];
    }
}

__device__ __forceinline__ Int4 multiply(const Int4 &w, const Int4 &x, const Int4 &acc) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
}

// Few outputs or tokens: a workgroup has OP x TP pieces of 16 outputs by 16 tokens, its wavefronts share the depth and
// add up through LDS.  Operands come straight from memory, kAhead steps of 64 inputs at once, overlapped with the
// products only where a workgroup has many of them (registers).  Bound by the weights' bytes: 16 tokens 5120 -> 13824
// 12.2 us (71 MB, 5.8 TB/s: of this size the cache behind the dies holds them between calls), and 3 for the codes.
template <typename T, int OP, int TP, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void shared_depth_kernel(const uint8_t *__restrict__ W,
                                                                  const uint8_t *__restrict__ X, int deep, int t_tiles,
                                                                  Scaled y) {
    constexpr int kAhead = OP + TP <= 3 ? 4 : 2;
    constexpr bool kOverlap = OP * TP >= 8;
    __shared__ Int4 red[WAVES][OP * TP][64];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int n = (int)die_order(blockIdx.x, gridDim.x);  // the token tiles of an output tile on one die
    const int64_t o0 = (int64_t)(n / t_tiles) * OP, t0 = (int64_t)(n % t_tiles) * TP;
    const int64_t last_o = (y.d_out - 1) / kRows, last_t = (y.m - 1) / kRows;
    const uint8_t *w[OP], *x[TP];
#pragma unroll
    for (int i = 0; i < OP; ++i) w[i] = W + min(o0 + i, last_o) * deep * kPiece + lane * 16;
#pragma unroll
    for (int i = 0; i < TP; ++i) x[i] = X + min(t0 + i, last_t) * deep * kPiece + lane * 16;
    // the scales that the results will take, on their way meanwhile
    constexpr int kMine = (OP * TP + WAVES - 1) / WAVES;
    const int64_t t = t0 * kRows + (lane & 15), o = o0 * kRows + (lane >> 4) * 4;
    float sx[kMine];
    float4 sw[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int q = wave + i * WAVES;
        sx[i] = token_scale(y, t + q % TP * kRows);
        sw[i] = output_scales(y, o + q / TP * kRows);
    }
    Int4 acc[OP][TP] = {};
    const int k0 = (int)((int64_t)deep * wave / WAVES), k1 = (int)((int64_t)deep * (wave + 1) / WAVES);
    Int4 a[2][kAhead][OP], b[2][kAhead][TP];
    auto load = [&](int k, int buf) {  // past the last step: that one again, which nothing multiplies
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = min(k + u, k1 - 1) * kPiece;
#pragma unroll
            for (int i = 0; i < OP; ++i) a[buf][u][i] = *reinterpret_cast<const Int4 *>(w[i] + at);
#pragma unroll
            for (int i = 0; i < TP; ++i) b[buf][u][i] = *reinterpret_cast<const Int4 *>(x[i] + at);
        }
    };
    auto compute = [&](int k, int buf) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k + u >= k1) break;
#pragma unroll
            for (int i = 0; i < OP; ++i)
#pragma unroll
                for (int j = 0; j < TP; ++j) acc[i][j] = multiply(a[buf][u][i], b[buf][u][j], acc[i][j]);
        }
    };
    if (!kOverlap) {
        for (int k = k0; k < k1; k += kAhead) {
            load(k, 0);
            compute(k, 0);
        }
    } else if (k0 < k1) {
        load(k0, 0);
        for (int k = k0; k < k1; k += 2 * kAhead) {
            load(k + kAhead, 1);
            compute(k, 0);
            load(k + 2 * kAhead, 0);
            compute(k + kAhead, 1);
        }
    }
#pragma unroll
    for (int i = 0; i < OP; ++i)
#pragma unroll
        for (int j = 0; j < TP; ++j) red[wave][i * TP + j][lane] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int q = wave + i * WAVES;
        if (q >= OP * TP) break;
        Int4 sum = red[0][q][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += red[v][q][lane];
        put4<T>(y, t + q % TP * kRows, o + q / TP * kRows, sum, sx[i], sw[i]);
    }
}

// One or two tokens in one launch: every workgroup codes the tokens for itself, 16 inputs a lane, while the first pieces
// of its 16 outputs' weights are on their way; the wavefronts share the depth.  Against coding them in a launch of
// its own, us: 1 token 8192 -> 1024 5.2 and 8.2, -> 28672 34.6 and 38.5; 2 tokens 8192 -> 8192 11.8 and 15.4; 4
// tokens 20.5 and 15.4, which is why it ends there.  Small ones are bound by what comes one after the other (the token,
// its largest, two barriers, the products, the join), large ones by the weights' bytes.
constexpr int kFewWaves = 16, kFewDepth = kFewWaves * 64 * 16;

template <typename TX, int M>
__global__ __launch_bounds__(kFewWaves * 64) void few_tokens_kernel(const uint8_t *__restrict__ W, const TX *__restrict__ X,
                                                                    int64_t d, int64_t ldx, int deep, Scaled y, int dtype,
                                                                    int32_t *__restrict__ status) {
    constexpr int kAhead = 4;
    __shared__ __align__(16) uint8_t codes[M * kFewDepth];
    __shared__ Int4 red[kFewWaves][64];
    __shared__ float most[M][kFewWaves], scales[M];
    const int lane = threadIdx.x & 63, wave = wave_index(), m = (int)y.m;
    const uint8_t *w = W + (int64_t)blockIdx.x * deep * kPiece + lane * 16;
    const int k0 = deep * wave / kFewWaves, k1 = deep * (wave + 1) / kFewWaves;
    Int4 a[kAhead];
    auto load = [&](int k) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) a[u] = *reinterpret_cast<const Int4 *>(w + (int64_t)min(k + u, deep - 1) * kPiece);
    };
    const int c = threadIdx.x, chunks = deep * 4;
    Sixteen<TX> x[M];
#pragma unroll
    for (int t = 0; t < M; ++t) x[t].load(X + min(t, m - 1) * ldx + c * 16, c < chunks ? d - c * 16 : 0);
    load(k0);
    bool bad = false;
#pragma unroll
    for (int t = 0; t < M; ++t) {
        Largest largest;
        x[t].look(largest);
        if (__ballot(largest.bad())) {
            bad = true;
            largest.bits = 0;
            x[t].look_again(largest);
        }
        float v = largest.most();
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s, CMPQ_WAVE));
        if (lane == 0) most[t][wave] = v;
    }
    if (bad && status && blockIdx.x == 0) atomicOr(status, CMPQ_STATUS_NONFINITE);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < M; ++t) {
        float v = most[t][0];
#pragma unroll
        for (int q = 1; q < kFewWaves; ++q) v = fmaxf(v, most[t][q]);
        const float s = code_scale(v), inv = 1.f / s;
        if (threadIdx.x == 0) scales[t] = s;
        if (c < chunks) *reinterpret_cast<uint4 *>(codes + t * kFewDepth + c * 16) = x[t].codes(inv, !bad);
    }
    __syncthreads();
    Int4 acc = {};
    const uint8_t *mine = codes + min(lane & 15, m - 1) * kFewDepth + (lane >> 4) * 16;
    for (int k = k0; k < k1; k += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k + u >= k1) break;
            acc = multiply(a[u], *reinterpret_cast<const Int4 *>(mine + (k + u) * kDepth), acc);
        }
        if (k + kAhead < k1) load(k + kAhead);
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll 5  // more at once would take the registers of a second workgroup a unit
    for (int v = 1; v < kFewWaves; ++v) acc += red[v][lane];
    const int64_t o = (int64_t)blockIdx.x * kRows + (lane >> 4) * 4;
    const float sx = scales[min(lane & 15, m - 1)];
    const float4 sw = output_scales(y, o);
    with_dtype(dtype, [&](auto like) { put4<decltype(like)>(y, lane & 15, o, acc, sx, sw); });
}

__device__ __forceinline__ void load_lds16(const uint8_t *src, uint8_t *dst) {
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) uint32_t *>(reinterpret_cast<uintptr_t>(src)),
                                     reinterpret_cast<__attribute__((address_space(3))) uint32_t *>((uint32_t)reinterpret_cast<uintptr_t>(dst)), 16, 0, 0);
}

// Tiles of OT x TT pieces a workgroup, WO x WT wavefronts.  Pieces reach LDS by direct loads in the order in which they
// are read (no conflicts), BUFS steps of 64 inputs in a ring; while a step is multiplied its operands are in
// registers, those of the next are on their way from LDS and the steps after it from memory.  Bound by the matrix
// instructions at 256 x 256: 4096 tokens 8192 -> 28672 in 741 us with the codes (29), 2.6 POP/s, the instructions busy for 69 %
// of the clocks, the rest at the barrier of a step.  64 x 64 (333 tokens 4099 -> 3001, 16 us): by what the caches deliver, 282 tiles
// of 66 steps of 8 KB, 9.4 TB/s; matrix instructions 14 %.  Bands keep the inputs of a die's tiles in its
// cache while the weights pass once a band.
constexpr int kBand = 4;

template <typename T, int OT, int TT, int WO, int WT, int BUFS>
__global__ __launch_bounds__(WO * WT * 64, 2) void tile_kernel(const uint8_t *__restrict__ W, const uint8_t *__restrict__ X,
                                                               int deep, int o_tiles, int t_tiles, Scaled y) {
    constexpr int kWaves = WO * WT, kLoads = (OT + TT) / kWaves, kStepBytes = (OT + TT) * kPiece, A = OT / WO, B = TT / WT;
    static_assert(kLoads * kWaves == OT + TT && A * WO == OT && B * WT == TT, "shares of the wavefronts");
    __shared__ __align__(16) uint8_t smem[BUFS * kStepBytes];
    const int lane = threadIdx.x & 63, wave = wave_index();
    // bands of kBand token tiles, all output tiles of a band one after the other
    const int64_t n = die_order(blockIdx.x, (int64_t)o_tiles * t_tiles);
    const int band = (int)(n / ((int64_t)kBand * o_tiles)), in_band = (int)(n - (int64_t)band * kBand * o_tiles);
    const int wide = min(kBand, t_tiles - band * kBand);
    const int64_t o0 = (int64_t)(in_band / wide) * OT, t0 = (int64_t)(band * kBand + in_band % wide) * TT;
    const int64_t last_o = (y.d_out - 1) / kRows, last_t = (y.m - 1) / kRows;
    const uint8_t *src[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int k = wave * kLoads + q;
        src[q] = (k < OT ? W + min(o0 + k, last_o) * deep * kPiece : X + min(t0 + k - OT, last_t) * deep * kPiece) + lane * 16;
    }
    uint8_t *dst = smem + wave * kLoads * kPiece;
    auto load = [&](int step, int q) {  // past the last step: that one again, which nothing reads
        load_lds16(src[q] + min(step, deep - 1) * kPiece, dst + (step % BUFS) * kStepBytes + q * kPiece);
    };
    const int wo = wave % WO * A, wt = wave / WO * B;
    Int4 acc[A][B] = {}, a[2][A], b[2][B];
    auto fetch = [&](int step, int buf, int q) {  // operand q of those of W, then of X
        const uint8_t *from = smem + (step % BUFS) * kStepBytes + lane * 16;
        if (q < A) a[buf][q] = *reinterpret_cast<const Int4 *>(from + (wo + q) * kPiece);
        else b[buf][q - A] = *reinterpret_cast<const Int4 *>(from + (OT + wt + q - A) * kPiece);
    };
    // This wavefront's loads of `step` have landed (those of BUFS - 2 later steps are under way) and its LDS reads have
    // returned.  After the barrier both hold for every wavefront: the step may be read, and the buffer of the one
    // before it loaded again.
    auto arrive = [&]() {
        constexpr int kUnder = (BUFS - 2) * kLoads;
        static_assert(kUnder < 64, "the count of loads still under way");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((kUnder & 15) | (kUnder >> 4) << 14 | 7 << 4);  // the same wait, for the compiler to count on
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kUnder) : "memory");
    };
    // Multiplies a step while the next one's operands come from LDS and a later one's pieces from memory, a share of
    // each at a time: issued together, the loads fill the memory pipeline's queue and hold up all behind them.
    auto turn = [&](int step, int buf) {
        arrive();
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
#pragma unroll
            for (int q = (A + B) * s / kLoads; q < (A + B) * (s + 1) / kLoads; ++q) fetch(step + 1, buf ^ 1, q);
#pragma unroll
            for (int i = A * B * s / kLoads; i < A * B * (s + 1) / kLoads; ++i) {
                acc[i / B][i % B] = multiply(a[buf][i / B], b[buf][i % B], acc[i / B][i % B]);
                if (i == A * B * (2 * s + 1) / (2 * kLoads)) load(step + BUFS, s);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int u = 0; u < BUFS - 1; ++u)
#pragma unroll
        for (int q = 0; q < kLoads; ++q) load(u, q);
    arrive();
#pragma unroll
    for (int q = 0; q < A + B; ++q) fetch(0, 0, q);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) load(BUFS - 1, q);
    for (int step = 0; step < deep; step += 2) {  // the depth is a multiple of two steps
        turn(step, 0);
        turn(step + 1, 1);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // what nothing reads ends before the LDS does
    const int64_t t = (t0 + wt) * kRows + (lane & 15), o = (o0 + wo) * kRows + (lane >> 4) * 4;
    float sx[B];
    float4 sw[A];
#pragma unroll
    for (int q = 0; q < B; ++q) sx[q] = token_scale(y, t + q * kRows);
#pragma unroll
    for (int p = 0; p < A; ++p) sw[p] = output_scales(y, o + p * kRows);
#pragma unroll
    for (int q = 0; q < B; ++q)
#pragma unroll
        for (int p = 0; p < A; ++p) put4<T>(y, t + q * kRows, o + p * kRows, acc[p][q], sx[q], sw[p]);
}

template <typename T, int OT, int TT, int WO, int WT, int BUFS>
void launch_tiles(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, hipStream_t st) {
    const int o_tiles = (int)cdiv(y.d_out, OT * kRows), t_tiles = (int)cdiv(y.m, TT * kRows);
    tile_kernel<T, OT, TT, WO, WT, BUFS><<<dim3((unsigned)(o_tiles * t_tiles)), WO * WT * 64, 0, st>>>(W, X, deep, o_tiles, t_tiles, y);
}

template <typename T, int OP, int TP, int WAVES>
void launch_shared(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, hipStream_t st) {
    const int64_t t_tiles = cdiv(y.m, TP * kRows), tiles = cdiv(y.d_out, OP * kRows) * t_tiles;
    shared_depth_kernel<T, OP, TP, WAVES><<<dim3((unsigned)tiles), WAVES * 64, 0, st>>>(W, X, deep, (int)t_tiles, y);
}

int64_t tiles_of(const Scaled &y, int ot, int tt) { return cdiv(y.d_out, ot * kRows) * cdiv(y.m, tt * kRows); }

// Which kernel: the largest tile that fills the chip.  A tile of 256 x 256 or 256 x 128 takes a compute unit for itself, so
// its last round has to be two thirds full, or one of many.  us (4096 tokens 8192 -> 28672; 2048 tokens 4096 -> 4096; 1024
// tokens 4096 -> 4096; 512 tokens 4096 -> 11008): 256 x 256 737, 60, 53, 53; 256 x 128 860, 43.1, 36, 34.8; 128 x 128 901,
// 44.0, 28, 35.4; 64 x 64 (333 tokens 4099 -> 3001 20.4, 128 x 128 25.5; 48 tokens 4096 -> 11008 14.0, 21.3).  Fewer than 150
// tiles of 64 x 64, and up to 32 tokens: wavefronts share the depth (512 tokens 8192 -> 1024 18.6, 64 x 64 23.0; 64 tokens
// 4096 -> 4096 9.4, 12.3).  Up to 16 tokens: two pieces of outputs a workgroup where there are many (16 tokens 5120 -> 13824
// 16.0, one piece 17.9), 8 wavefronts for some (8192 -> 8192 15.8, 16 wavefronts 16.4), 16 for few (8 tokens 8192 -> 1024
// 8.6, 8 wavefronts 9.8).
template <typename T>
int launch_product(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, hipStream_t st) {
    constexpr int64_t kUnits = 256;  // compute units
    auto fills = [](int64_t n) { return n >= 4 * kUnits || (n + kUnits / 3) / kUnits * kUnits >= n; };  // 171 .. 256, 427 .. 512, ...
    const int64_t pieces = cdiv(y.d_out, kRows);
    if (tiles_of(y, 1, 1) > INT32_MAX) return CMPQ_ESHAPE;
    if (y.m <= 16 && pieces >= 768) launch_shared<T, 2, 1, 8>(W, X, deep, y, st);
    else if (y.m <= 16 && pieces >= 320) launch_shared<T, 1, 1, 8>(W, X, deep, y, st);
    else if (y.m <= 16) launch_shared<T, 1, 1, 16>(W, X, deep, y, st);
    else if (y.m <= 32) launch_shared<T, 4, 2, 4>(W, X, deep, y, st);
    else if (fills(tiles_of(y, 16, 16))) launch_tiles<T, 16, 16, 4, 2, 4>(W, X, deep, y, st);
    else if (fills(tiles_of(y, 16, 8))) launch_tiles<T, 16, 8, 4, 2, 4>(W, X, deep, y, st);
    else if (tiles_of(y, 8, 8) >= 192) launch_tiles<T, 8, 8, 2, 2, 4>(W, X, deep, y, st);
    else if (tiles_of(y, 4, 4) >= 150) launch_tiles<T, 4, 4, 2, 2, 8>(W, X, deep, y, st);
    else launch_shared<T, 4, 2, 4>(W, X, deep, y, st);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

template <typename TX>
void launch_few(const uint8_t *W, const void *X, int64_t d, int64_t ldx, const Scaled &y, int y_dtype, int32_t *status,
                hipStream_t st) {
    const dim3 grid((unsigned)cdiv(y.d_out, kRows));
    const TX *x = static_cast<const TX *>(X);
    const int deep = (int)pieces_deep(d);
    if (y.m == 1) few_tokens_kernel<TX, 1><<<grid, kFewWaves * 64, 0, st>>>(W, x, d, ldx, deep, y, y_dtype, status);
    else few_tokens_kernel<TX, 2><<<grid, kFewWaves * 64, 0, st>>>(W, x, d, ldx, deep, y, y_dtype, status);
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
    const size_t four = 4 * dtype_bytes(y_dtype);
    const Scaled y = {w.scale, scale, Y, m, d_out, ldy,
                      ldy % 4 == 0 && reinterpret_cast<uintptr_t>(Y) % four == 0 && reinterpret_cast<uintptr_t>(scale) % 16 == 0};
    const uint8_t *cw = reinterpret_cast<const uint8_t *>(codes), *cx = reinterpret_cast<const uint8_t *>(w.codes);
    if (m <= 2 && d_in <= kFewDepth) {
        if (dtype == CMPQ_F16) launch_few<_Float16>(cw, X, d_in, ldx, y, y_dtype, status, st);
        else if (dtype == CMPQ_BF16) launch_few<__bf16>(cw, X, d_in, ldx, y, y_dtype, status, st);
        else launch_few<float>(cw, X, d_in, ldx, y, y_dtype, status, st);
        CMPQ_LAUNCH_CHECK();
        return CMPQ_OK;
    }
    if (int rc = launch_code_rows_of(X, dtype, m, d_in, ldx, m, w.codes, w.scale, status, st)) return rc;
    const int deep = (int)pieces_deep(d_in);
    if (y_dtype == CMPQ_F16) return launch_product<_Float16>(cw, cx, deep, y, st);
    if (y_dtype == CMPQ_BF16) return launch_product<__bf16>(cw, cx, deep, y, st);
    return launch_product<float>(cw, cx, deep, y, st);
}
