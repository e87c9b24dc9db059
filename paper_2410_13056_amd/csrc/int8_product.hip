// Products in 8-bit integers: codes with a scale per row of either operand, exact sums, one multiplication by each
// scale at the end, and what may follow it (epilogue.h).
#include "epilogue.h"
#include "int8_rows.h"

namespace {

typedef int32_t Int4 __attribute__((ext_vector_type(4)));

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

// Rows come in groups of 16; this operand's is every `of`-th of them, from `at` on.
struct Turn {
    int of, at;
};

// One row a workgroup, or four in turn from lane to lane: the row's largest magnitude, then its codes, 16 inputs a lane and step.
// Rows of up to KEPT * THREADS / ROWS * 16 inputs stay in registers between the two, longer ones are read again.  Rows from n to
// `all` are zeros.
//
// The rows of a piece write 16 bytes each of the same lines, so consecutive rows go to one die, whose cache puts the lines together.
// Bound by bytes where rows are many, and then by the number of runs that the stores come in (one of 1 KB each in place of 64 of 16
// bytes: 38 us where it is 47 for 2048 rows of 28672): four rows together write 64 bytes in order.  4096 rows of 8192 from memory 26 us, 3.9
// TB/s, one by one 29.8, 2048 of 13824 22.1 and 26.8; from the cache behind the dies the same, and fewer rows are better off one by one, 1280
// of 8192 7.2 and 8.9.  Bound by a row's latency where they are few: 333 rows 4 us.  Long rows take 16 wavefronts in place of 4: 2048 of
// 28672 from memory 47 us and 55 (34 and 32 from the cache), 300 of 28672 8.0 and 8.5, 1 of 28672 5.1 and 6.3, 16 of 13824 4.7 and 5.2,
// but 1 of 8192 4.1 and 3.6.  Lines: rows of 13824 by 16 and by 4, 192 rows 4.5 and 5.2, 256 4.9 and 5.3, 320 5.5 and 5.8, 512 6.5 and 6.6, 768 8.6 and
// 8.1; rows of 8192 one by one and four together, from memory 1280 10.9 and 11.4, 1792 14.5 and 12.7, 2048 16.1 and 13.8, 4096 29.0 and 25.5 (from
// the caches 7.2 and 8.8, 10.5 and 10.4, 12.1 and 11.0, 19.4 and 19.6).
template <typename T, int THREADS, int KEPT, int ROWS>
__global__ __launch_bounds__(THREADS) void code_rows_kernel(const T *__restrict__ X, int64_t n, int64_t all, int64_t d, int64_t ld,
                                                        int8_t *__restrict__ codes, float *__restrict__ scale, Turn turn,
                                                        int32_t *__restrict__ status) {
    constexpr int kLanes = THREADS / ROWS;  // of a row
    static_assert(ROWS == 1 || (ROWS == 4 && THREADS == 1024), "what four_rows_max joins");
    __shared__ float scratch[THREADS / 64 * ROWS];
    const int64_t row = die_order(blockIdx.x, gridDim.x) * ROWS + threadIdx.x % ROWS, deep = pieces_deep(d);
    const int64_t group = row / kRows * turn.of + turn.at;
    const int first = threadIdx.x / ROWS, groups = row < all ? (int)deep * 4 : 0;
    const int64_t valid = row < n ? d : 0;
    uint8_t *out = reinterpret_cast<uint8_t *>(codes) + group * deep * kPiece + row % kRows * 16;
    const T *x = X + row * ld;
    Largest largest;
    Sixteen<T> kept[KEPT > 0 ? KEPT : 1];
    auto each = [&](auto fn) {  // fn(sixteen inputs, their number), from registers where they were kept
        if (KEPT > 0) {
#pragma unroll
            for (int k = 0; k < KEPT; ++k)
                if (first + k * kLanes < groups) fn(kept[k], first + k * kLanes);
        } else {
            for (int c = first; c < groups; c += kLanes) {
                kept[0].load(x + c * 16, valid - c * 16);
                fn(kept[0], c);
            }
        }
    };
    if (KEPT > 0) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            const int c = first + k * kLanes;
            kept[k].load(x + c * 16, c < groups ? valid - c * 16 : 0);
        }
    }
    each([&](const Sixteen<T> &s, int) { s.look(largest); });
    const bool bad = __ballot(largest.bad()) != 0;
    if (bad) {
        largest.bits = 0;
        each([&](const Sixteen<T> &s, int) { s.look_again(largest); });
        if (status) atomicOr(status, CMPQ_STATUS_NONFINITE);
    }
    float most;
    if constexpr (ROWS == 1) most = block_max(largest.most(), scratch);
    else most = four_rows_max(largest.most(), scratch);
    const float s = code_scale(most), inv = 1.f / s;
    if (first == 0 && row < all) {
        if (row < n) scale[group * kRows + row % kRows] = s;
        else if (turn.of > 1) scale[group * kRows + row % kRows] = 0.f;
    }
    auto put = [&](const Sixteen<T> &s, int c, bool clean) {
        *reinterpret_cast<uint4 *>(out + c / 4 * kPiece + c % 4 * 256) = s.codes(inv, clean);
    };
    if (bad) each([&](const Sixteen<T> &s, int c) { put(s, c, false); });
    else each([&](const Sixteen<T> &s, int c) { put(s, c, true); });
}

template <int N>
using Kept = std::integral_constant<int, N>;

template <typename T>
void launch_code_rows(const void *X, int64_t n, int64_t d, int64_t ld, int64_t rows, int8_t *codes, float *scale,
                      Turn turn, int32_t *status, hipStream_t st) {
    const T *x = static_cast<const T *>(X);
    const auto run = [&](auto threads, auto kept, auto together) {
        for (int64_t at = 0; at < rows; at += kRowsOfLaunch) {
            const int64_t here = rows - at < kRowsOfLaunch ? rows - at : kRowsOfLaunch;
            code_rows_kernel<T, threads(), kept(), together()><<<dim3((unsigned)cdiv(here, together())), threads(), 0, st>>>(
                x + at * ld, n - at, here, d, ld, codes + at / kRows * turn.of * pieces_deep(d) * kPiece, scale + at * turn.of, turn, status);
        }
    };
    typedef std::integral_constant<int, 256> Four;  // wavefronts
    typedef std::integral_constant<int, 1024> Many;
    typedef std::integral_constant<int, 1> One;  // row
    typedef std::integral_constant<int, 4> Rows;
    const bool few = rows <= 256, many = rows >= 2048;
    if (d <= 4096 && many) run(Many(), Kept<1>(), Rows());
    else if (d <= 4096) run(Four(), Kept<1>(), One());
    else if (d <= 8192 && many) run(Many(), Kept<2>(), Rows());
    else if (d <= 8192) run(Four(), Kept<2>(), One());
    else if (d <= 16384 && many) run(Many(), Kept<4>(), Rows());
    else if (d <= 16384 && few) run(Many(), Kept<1>(), One());
    else if (d <= 16384) run(Four(), Kept<4>(), One());
    else if (d <= 32768) run(Many(), Kept<2>(), One());
    else run(Four(), Kept<0>(), One());
}

// `rows` of them, those from n on zeros.
int launch_code_rows_of(const void *X, int dtype, int64_t n, int64_t d, int64_t ld, int64_t rows, int8_t *codes,
                     float *scale, Turn turn, int32_t *status, hipStream_t st) {
    if (dtype == CMPQ_F16) launch_code_rows<_Float16>(X, n, d, ld, rows, codes, scale, turn, status, st);
    else if (dtype == CMPQ_BF16) launch_code_rows<__bf16>(X, n, d, ld, rows, codes, scale, turn, status, st);
    else launch_code_rows<float>(X, n, d, ld, rows, codes, scale, turn, status, st);
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

// What follows the scaled sums.  The kernels come without anything behind them, with an epilogue, and gated: pieces of 16
// outputs of the gate and of the second factor in turn, so that the wavefront that has the one has the other.
struct Plain {
    static constexpr bool kPlain = true, kGated = false;
};
struct Epilogue {
    static constexpr bool kPlain = false, kGated = false;
    const void *bias, *up_bias, *residual;
    int64_t ldr;
    int bias_dtype, r_dtype, y_dtype, act;
};
struct GatedEpilogue : Epilogue {
    static constexpr bool kGated = true;
};
template <typename E>
constexpr int kPerOutput = E::kGated ? 2 : 1;  // rows of the weight that make an output

// N outputs o, o + 1, ... of token t, `n` of them there, from their scaled sums v (and u, the second factor's); b: biases
template <typename E, int N>
__device__ __forceinline__ void finish(const Scaled &y, const E &e, int64_t t, int64_t o, int n, float (&v)[N],
                                       const float (&u)[N], const float (&b)[N], const float (&bu)[N]) {
#pragma clang fp contract(off)
    float r[N];
    if (e.residual) load_some<N>(e.residual, e.r_dtype, t * e.ldr + o, n, r);
    if (e.bias) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += b[i];
    }
    activate(e.act, v);
    if (E::kGated) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= e.up_bias ? u[i] + bu[i] : u[i];
    }
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += r[i];
    }
    store_some<N>(y.Y, e.y_dtype, t * y.ldy + o, n, v);
}

// Scales of a weight's rows and biases of N outputs from o on, `n` of them there.
template <typename E, int N>
struct Columns {
    float sw[N], su[N], b[N], bu[N];
    __device__ __forceinline__ void load(const Scaled &y, const E &e, int64_t o, int n) {
        if (E::kGated) {  // whole pieces of either
            const float *s = y.sw + o / kRows * (2 * kRows) + o % kRows;
            load_f32<float, N>(s, sw);
            load_f32<float, N>(s + kRows, su);
        } else {
            load_some<N>(y.sw, CMPQ_F32, o, n, sw);
        }
        if (e.bias) load_some<N>(e.bias, e.bias_dtype, o, n, b);
        if (E::kGated && e.up_bias) load_some<N>(e.up_bias, e.bias_dtype, o, n, bu);
    }
};

// Outputs o .. o + 3 of token t with everything that follows the sums.
template <typename T, typename E>
__device__ __forceinline__ void put_finished(const Scaled &y, const E &e, int64_t t, int64_t o, const Int4 &acc, const Int4 &up, float sx) {
    const int n = (int)min(y.d_out - o, (int64_t)4);
    if (t >= y.m || n <= 0) return;
    Columns<E, 4> c;
    c.load(y, e, o, n);
    float v[4], u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = scaled(acc[i], sx, c.sw[i]);
        if (E::kGated) u[i] = scaled(up[i], sx, c.su[i]);
    }
    finish<E, 4>(y, e, t, o, n, v, u, c.b, c.bu);
}

__device__ __forceinline__ Int4 multiply(const Int4 &w, const Int4 &x, const Int4 &acc) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
}

// Few outputs or tokens: a workgroup has OP x TP pieces of 16 outputs by 16 tokens, its wavefronts share the depth and
// add up through LDS.  Operands come straight from memory, kAhead steps of 64 inputs at once, overlapped with the
// products only where a workgroup has many of them (registers).  A step in turn for each wavefront and not a run of steps: 4 tokens
// 28672 -> 8192, weights from memory, 44 us and 49, 16 tokens 13824 -> 5120 19.9 and 20.8.  Bound by the weights' bytes: 16 tokens 5120 -> 13824
// 12.2 us (71 MB, 5.8 TB/s: of this size the cache behind the dies holds them between calls), and 3 for the codes.
template <typename T, typename E, int OP, int TP, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void shared_depth_kernel(const uint8_t *__restrict__ W,
                                                                  const uint8_t *__restrict__ X, int deep, int t_tiles,
                                                                  Scaled y, E e) {
    constexpr int kAhead = OP + TP <= 3 ? 4 : 2;
    constexpr bool kOverlap = OP * TP >= 8;
    __shared__ Int4 red[WAVES][OP * TP][64];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int n = (int)die_order(blockIdx.x, gridDim.x);  // the token tiles of an output tile on one die
    const int64_t o0 = (int64_t)(n / t_tiles) * OP, t0 = (int64_t)(n % t_tiles) * TP;
    const int64_t last_o = ((y.d_out - 1) / kRows + 1) * kPerOutput<E> - 1, last_t = (y.m - 1) / kRows;
    const uint8_t *w[OP], *x[TP];
#pragma unroll
    for (int i = 0; i < OP; ++i) w[i] = W + min(o0 + i, last_o) * deep * kPiece + lane * 16;
#pragma unroll
    for (int i = 0; i < TP; ++i) x[i] = X + min(t0 + i, last_t) * deep * kPiece + lane * 16;
    // the scales that the results will take, on their way meanwhile
    static_assert(OP % kPerOutput<E> == 0, "pieces of an output in one workgroup");
    constexpr int kResults = OP / kPerOutput<E> * TP, kMine = (kResults + WAVES - 1) / WAVES;
    const int64_t t = t0 * kRows + (lane & 15), o = o0 / kPerOutput<E> * kRows + (lane >> 4) * 4;
    float sx[kMine];
    float4 sw[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int q = wave + i * WAVES;
        sx[i] = token_scale(y, t + q % TP * kRows);
        if (E::kPlain) sw[i] = output_scales(y, o + q / TP * kRows);
    }
    Int4 acc[OP][TP] = {};
    const int steps = (deep - wave + WAVES - 1) / WAVES;  // of the wavefront: every WAVES-th, so that they read next to each other
    Int4 a[2][kAhead][OP], b[2][kAhead][TP];
    auto load = [&](int k, int buf) {  // past the last step: that one again, which nothing multiplies
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = (min(k + u, steps - 1) * WAVES + wave) * kPiece;
#pragma unroll
            for (int i = 0; i < OP; ++i) a[buf][u][i] = *reinterpret_cast<const Int4 *>(w[i] + at);
#pragma unroll
            for (int i = 0; i < TP; ++i) b[buf][u][i] = *reinterpret_cast<const Int4 *>(x[i] + at);
        }
    };
    auto compute = [&](int k, int buf) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k + u >= steps) break;
#pragma unroll
            for (int i = 0; i < OP; ++i)
#pragma unroll
                for (int j = 0; j < TP; ++j) acc[i][j] = multiply(a[buf][u][i], b[buf][u][j], acc[i][j]);
        }
    };
    if (!kOverlap) {
        for (int k = 0; k < steps; k += kAhead) {
            load(k, 0);
            compute(k, 0);
        }
    } else if (steps > 0) {
        load(0, 0);
        for (int k = 0; k < steps; k += 2 * kAhead) {
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
        if (q >= kResults) break;
        auto total = [&](int p) {
            Int4 sum = red[0][p][lane];
#pragma unroll(E::kPlain ? WAVES : 4)
            for (int v = 1; v < WAVES; ++v) sum += red[v][p][lane];
            return sum;
        };
        const int64_t tq = t + q % TP * kRows, oq = o + q / TP * kRows;
        if constexpr (E::kPlain) {
            put4<T>(y, tq, oq, total(q), sx[i], sw[i]);
        } else {
            const int p = q / TP * kPerOutput<E> * TP + q % TP;  // the gate's result; the second factor's is TP further on
            put_finished<T, E>(y, e, tq, oq, total(p), E::kGated ? total(p + TP) : Int4{}, sx[i]);
        }
    }
}

// One or two tokens in one launch: every workgroup codes the tokens for itself, 16 inputs a lane, while the first pieces
// of its 16 outputs' weights are on their way; the wavefronts share the depth.  Against coding them in a launch of
// its own, us: 1 token 8192 -> 1024 5.2 and 8.2, -> 28672 34.6 and 38.5, 28672 -> 8192 37.7 and 41.6, -> 512 9.1 and 18.6; 2 tokens
// 8192 -> 8192 11.8 and 15.4, 28672 -> 1000 12.0 and 19.4, -> 4000 23.6 and 27.0 (a gated product's second token of more
// than 16384 inputs has no room in registers); 4 tokens 20.5 and 15.4, which is why it ends there.  Small ones are bound by what comes one after the other (the
// token, its largest, two barriers, the products, the join), large ones by the weights' bytes.
// Wavefronts: eight_wavefronts; 1 token 8192 -> 28672 36.3 us with 8 and 34.8 with 16; gated, weights from memory, 5120 -> 2 x 13824
// 29.8 and 29.6, 8192 -> 2 x 28672 86.6 and 85.0 (5.5 TB/s; loads alone in runs of 128 KB reach 6.2).  A step in turn for each
// wavefront in place of a run of steps: gated 85.0 and 90, but 8192 -> 28672 42.8 and 41.7.
constexpr int kFewDepth = 16384;

template <typename TX, typename E, int M, int C, int WAVES>  // up to C * 1024 * WAVES inputs
__global__ __launch_bounds__(WAVES * 64) void few_tokens_kernel(const uint8_t *__restrict__ W, const TX *__restrict__ X,
                                                                    int64_t d, int64_t ldx, int deep, Scaled y, E e, int dtype,
                                                                    int32_t *__restrict__ status) {
    constexpr int kAhead = 4, P = kPerOutput<E>, kMost = C * WAVES * 1024;
    __shared__ __align__(16) uint8_t codes[M * kMost];
    __shared__ Int4 red[P][WAVES][64];
    __shared__ float most[M][WAVES], scales[M];
    const int lane = threadIdx.x & 63, wave = wave_index(), m = (int)y.m;
    const uint8_t *w = W + (int64_t)blockIdx.x * P * deep * kPiece + lane * 16;
    // Steps of the wavefront: gated, every WAVES-th, else a run of them.
    const int first = E::kGated ? wave : deep * wave / WAVES, apart = E::kGated ? WAVES : 1;
    const int steps = E::kGated ? (deep - wave + WAVES - 1) / WAVES : deep * (wave + 1) / WAVES - first;
    Int4 a[kAhead][P];
    // Past the wavefront's steps: with 8 wavefronts nothing, where that would be much of its loads; else the last bytes again, which
    // nothing multiplies: that costs less there than to ask.
    constexpr bool kAsk = WAVES == 8;
    auto load = [&](int k) {
        const bool all = k + kAhead <= steps;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (kAsk && !all && k + u >= steps) break;
            const int at = min(first + (k + u) * apart, deep - 1);
#pragma unroll
            for (int p = 0; p < P; ++p) a[u][p] = *reinterpret_cast<const Int4 *>(w + ((int64_t)p * deep + at) * kPiece);
        }
    };
    const int chunks = deep * 4;
    const auto chunk = [&](int i) { return (int)threadIdx.x + i * (WAVES * 64); };
    Sixteen<TX> x[M][C];
#pragma unroll
    for (int t = 0; t < M; ++t)
#pragma unroll
        for (int i = 0; i < C; ++i) x[t][i].load(X + min(t, m - 1) * ldx + chunk(i) * 16, chunk(i) < chunks ? d - chunk(i) * 16 : 0);
    load(0);
    bool bad = false;
#pragma unroll
    for (int t = 0; t < M; ++t) {
        Largest largest;
#pragma unroll
        for (int i = 0; i < C; ++i) x[t][i].look(largest);
        if (__ballot(largest.bad())) {
            bad = true;
            largest.bits = 0;
#pragma unroll
            for (int i = 0; i < C; ++i) x[t][i].look_again(largest);
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
        for (int q = 1; q < WAVES; ++q) v = fmaxf(v, most[t][q]);
        const float s = code_scale(v), inv = 1.f / s;
        if (threadIdx.x == 0) scales[t] = s;
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (chunk(i) < chunks) *reinterpret_cast<uint4 *>(codes + t * (kMost) + chunk(i) * 16) = x[t][i].codes(inv, !bad);
    }
    __syncthreads();
    Int4 acc[P] = {};
    const uint8_t *mine = codes + min(lane & 15, m - 1) * (kMost) + (lane >> 4) * 16;
    for (int k = 0; k < steps; k += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k + u >= steps) break;
            const Int4 b = *reinterpret_cast<const Int4 *>(mine + (first + (k + u) * apart) * kDepth);
#pragma unroll
            for (int p = 0; p < P; ++p) acc[p] = multiply(a[u][p], b, acc[p]);
        }
        if (k + kAhead < steps) load(k + kAhead);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) red[p][wave][lane] = acc[p];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll 5  // more at once would take the registers of a second workgroup a unit
    for (int v = 1; v < WAVES; ++v)
#pragma unroll
        for (int p = 0; p < P; ++p) acc[p] += red[p][v][lane];
    const int64_t o = (int64_t)blockIdx.x * kRows + (lane >> 4) * 4;
    const float sx = scales[min(lane & 15, m - 1)];
    if constexpr (E::kPlain) {
        const float4 sw = output_scales(y, o);
        with_dtype(dtype, [&](auto like) { put4<decltype(like)>(y, lane & 15, o, acc[0], sx, sw); });
    } else {
        put_finished<float, E>(y, e, lane & 15, o, acc[0], acc[P - 1], sx);
    }
}

__device__ __forceinline__ void load_lds16(const uint8_t *src, uint8_t *dst) {
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) uint32_t *>(reinterpret_cast<uintptr_t>(src)),
                                     reinterpret_cast<__attribute__((address_space(3))) uint32_t *>((uint32_t)reinterpret_cast<uintptr_t>(dst)), 16, 0, 0);
}

// Sums of a wavefront on their way through LDS, a token's 16 A next to each other: where four of them (`four` < 4 A) of a row
// lie.  The rows of one store, and the fours of one load, go to different banks.
template <int A>
__device__ __forceinline__ int staged_sum(int row, int four) {
    return row * (A * 4) + (four ^ (row & (A * 4 - 1)));
}
// Pieces of 16 tokens that the wavefronts stage at once.
constexpr int tokens_at_once(int a, int b, int waves, int bytes) {
    while (b * a * 1024 * waves > bytes) b /= 2;
    return b;
}

// Finishes staged sums: ROWS tokens from t0 on, outputs from o0 on, eight outputs a lane, so that residuals and
// outputs pass in runs of whole lines and the code behind the sums is there once.
template <typename E, int A, int ROWS>
__device__ __forceinline__ void finish_rows(const Int4 *sums, const Scaled &y, const E &e, int64_t t0, int64_t o0) {
    constexpr int kLanes = A * 2 / kPerOutput<E>, kRowsAtOnce = 64 / kLanes;  // lanes that share a token
    const int lane = threadIdx.x & 63, j = lane % kLanes;
    const int64_t o = o0 + j * 8;
    const int n = (int)min(y.d_out - o, (int64_t)8);
    if (n <= 0) return;
    Columns<E, 8> c;
    c.load(y, e, o, n);
    const int first = E::kGated ? j / 2 * 8 + j % 2 * 2 : j * 2;
#pragma unroll 2
    for (int row = lane / kLanes; row < ROWS; row += kRowsAtOnce) {
        const int64_t t = t0 + row;
        if (t >= y.m) break;
        const float sx = y.sx[t];
        float v[8], u[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Int4 a = sums[staged_sum<A>(row, first + h)];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = scaled(a[i], sx, c.sw[4 * h + i]);
            if (E::kGated) {
                const Int4 b = sums[staged_sum<A>(row, first + 4 + h)];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[4 * h + i] = scaled(b[i], sx, c.su[4 * h + i]);
            }
        }
        finish<E, 8>(y, e, t, o, n, v, u, c.b, c.bu);
    }
}

// Staged sums with nothing behind them, for outputs that put4 would write one by one; its bits.
template <typename T, int A, int ROWS>
__device__ __forceinline__ void put_rows(const Int4 *sums, const Scaled &y, int64_t t0, int64_t o0) {
    constexpr int kLanes = A * 2, kRowsAtOnce = 64 / kLanes;  // lanes that share a token
    typedef T V __attribute__((ext_vector_type(8)));
    typedef V Any __attribute__((aligned(sizeof(T))));
    const int lane = threadIdx.x & 63, j = lane % kLanes;
    const int64_t o = o0 + j * 8;
    const int n = (int)min(y.d_out - o, (int64_t)8);
    if (n <= 0) return;
    float sw[8];
    load_some<8>(y.sw, CMPQ_F32, o, n, sw);
    for (int row = lane / kLanes; row < ROWS; row += kRowsAtOnce) {
        const int64_t t = t0 + row;
        if (t >= y.m) break;
        const float sx = y.sx[t];
        V v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Int4 a = sums[staged_sum<A>(row, 2 * j + h)];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = (T)scaled(a[i], sx, sw[4 * h + i]);
        }
        T *p = static_cast<T *>(y.Y) + t * y.ldy + o;
        if (n == 8) {
            *reinterpret_cast<Any *>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = v[i];
        }
    }
}

// Tiles of OT x TT pieces a workgroup, WO x WT wavefronts.  Pieces reach LDS by direct loads in the order in which they
// are read (no conflicts), BUFS steps of 64 inputs in a ring; while a step is multiplied its operands are in
// registers, those of the next are on their way from LDS and the steps after it from memory.  Bound by the matrix
// instructions at 256 x 256: 4096 tokens 8192 -> 28672 in 690 us, and 24 for the codes (cards differ by 5 %), 2.8 POP/s, the
// instructions busy for 70 % of the clocks; on another day without the barriers 690 in place of 718 us, without the loads 626, without the LDS reads 677.  G groups of
// wavefronts share the depth, each with a ring of its own; their sums are joined through LDS, in order.  One round of small tiles: 3 us
// of a launch, 2 to 5 before the first step and behind the last, then 80 to 120 ns a step of 64 x 64 (of 118 bytes a ns that a unit's
// loads reach 70 to 100), 160 of 64 x 128, 230 of 128 x 128; without loads, without LDS reads or without barriers 0 to 15 % less.
// More buffers, or steps in another order a workgroup, change nothing.  Bands keep the inputs of a die's tiles in its
// cache while the weights pass once a band.
constexpr int kBand = 4;

template <typename T, typename E, int OT, int TT, int WO, int WT, int G, int BUFS, bool BEHIND_FIRST>
__global__ __launch_bounds__(WO * WT * G * 64, 2) void tile_kernel(const uint8_t *__restrict__ W, const uint8_t *__restrict__ X,
                                                               int deep, int o_tiles, int t_tiles, Scaled y, E e) {
    constexpr int kWaves = WO * WT, kLoads = (OT + TT) / kWaves, kStepBytes = (OT + TT) * kPiece, A = OT / WO, B = TT / WT;
    static_assert(kLoads * kWaves == OT + TT && A * WO == OT && B * WT == TT, "shares of the wavefronts");
    static_assert((G - 1) * OT * TT <= G * BUFS * (OT + TT), "room for the sums that are joined");
    __shared__ __align__(16) uint8_t smem[G * BUFS * kStepBytes];
    const int lane = threadIdx.x & 63, wave = G > 1 ? wave_index() % kWaves : wave_index(), group = G > 1 ? wave_index() / kWaves : 0;
    const int each = G > 1 ? (deep / 2 + G - 1) / G * 2 : deep;  // steps of a group, the last one's perhaps fewer
    const int from = group * each, mine = G > 1 ? min(each, deep - from) : deep;
    // bands of kBand token tiles, all output tiles of a band one after the other
    const int64_t n = die_order(blockIdx.x, (int64_t)o_tiles * t_tiles);
    const int band = (int)(n / ((int64_t)kBand * o_tiles)), in_band = (int)(n - (int64_t)band * kBand * o_tiles);
    const int wide = min(kBand, t_tiles - band * kBand);
    const int64_t o0 = (int64_t)(in_band / wide) * OT, t0 = (int64_t)(band * kBand + in_band % wide) * TT;
    const int64_t last_o = ((y.d_out - 1) / kRows + 1) * kPerOutput<E> - 1, last_t = (y.m - 1) / kRows;
    const uint8_t *src[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int k = wave * kLoads + q;
        src[q] = (k < OT ? W + min(o0 + k, last_o) * deep * kPiece : X + min(t0 + k - OT, last_t) * deep * kPiece) + lane * 16;
    }
    uint8_t *ring = smem + group * (BUFS * kStepBytes), *dst = ring + wave * kLoads * kPiece;
    auto load = [&](int step, int q) {  // past the last step: that one again, which nothing reads
        load_lds16(src[q] + min(from + step, deep - 1) * kPiece, dst + (step % BUFS) * kStepBytes + q * kPiece);
    };
    const int wo = wave % WO * A, wt = wave / WO * B;
    Int4 acc[A][B] = {}, a[2][A], b[2][B];
    auto fetch = [&](int step, int buf, int q) {  // operand q of those of W, then of X
        const uint8_t *at = ring + (step % BUFS) * kStepBytes + lane * 16;
        if (q < A) a[buf][q] = *reinterpret_cast<const Int4 *>(at + (wo + q) * kPiece);
        else b[buf][q - A] = *reinterpret_cast<const Int4 *>(at + (OT + wt + q - A) * kPiece);
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
        // The two wavefronts of a SIMD are seldom as far as each other: the one that is behind goes first until its last share.  4096
        // tokens 8192 -> 28672 747 us and 757, gated 1452 and 1482; raised for half of a step 750, for all of it 757.
        // Not for tiles of 128 x 128 that are more than two a unit: 700 tokens 13824 -> 13824 171 us without, 186 with; but 333 tokens
        // 8192 -> 11008, 258 tiles, 54 and 49.
        if (BEHIND_FIRST) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
            if (BEHIND_FIRST && s == kLoads - 1) __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int q = (A + B) * s / kLoads; q < (A + B) * (s + 1) / kLoads; ++q) fetch(step + 1, buf ^ 1, q);
#pragma unroll
            for (int i = A * B * s / kLoads; i < A * B * (s + 1) / kLoads; ++i) {
                if (G == 1 || step < mine) acc[i / B][i % B] = multiply(a[buf][i / B], b[buf][i % B], acc[i / B][i % B]);
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
    for (int step = 0; step < each; step += 2) {  // the depth is a multiple of two steps
        turn(step, 0);
        turn(step + 1, 1);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // what nothing reads ends before the LDS does
    // The groups' sums are joined through LDS, in order; each group finishes its share of the tokens.
    constexpr int kOwn = B / G;
    static_assert(kOwn * G == B, "tokens of a group");
    Int4 own[A][kOwn];
    if constexpr (G == 1) {
#pragma unroll
        for (int i = 0; i < A * B; ++i) own[i / B][i % B] = acc[i / B][i % B];
    } else {
        constexpr int kPart = A * kOwn * 64;
        __syncthreads();
        Int4 *sums = reinterpret_cast<Int4 *>(smem);  // [finishing group][wavefront][other group]
#pragma unroll
        for (int g = 0; g < G; ++g) {
            Int4 *to = sums + ((g * kWaves + wave) * (G - 1) + (group < g ? group : group - 1)) * kPart + lane;
#pragma unroll
            for (int i = 0; i < A * kOwn; ++i) {
                if (group == g) own[i / kOwn][i % kOwn] = acc[i / kOwn][g * kOwn + i % kOwn];
                else to[i * 64] = acc[i / kOwn][g * kOwn + i % kOwn];
            }
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < G - 1; ++g) {
            const Int4 *from = sums + ((group * kWaves + wave) * (G - 1) + g) * kPart + lane;
#pragma unroll
            for (int i = 0; i < A * kOwn; ++i) own[i / kOwn][i % kOwn] += from[i * 64];
        }
    }
    const int64_t t_own = t0 + wt + group * kOwn;
    // Plain outputs too where they cannot be written four at once: 333 tokens 4099 -> 3001 in FP16 11.7 us, one by one 12.8; 700 tokens
    // 1000 -> 3001 9.0 and 11.6; 2048 tokens 4096 -> 4097 49 and 61.
    if (!E::kPlain || !y.aligned) {
        __syncthreads();  // nobody's loads or sums are under way in the LDS that the results pass through now
        constexpr int kAtOnce = tokens_at_once(A, kOwn, kWaves * G, G * BUFS * kStepBytes);
        Int4 *through = reinterpret_cast<Int4 *>(smem) + (group * kWaves + wave) * (kAtOnce * A * 64);
#pragma unroll
        for (int q0 = 0; q0 < kOwn; q0 += kAtOnce) {
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q)
#pragma unroll
                for (int p = 0; p < A; ++p) through[staged_sum<A>(q * kRows + (lane & 15), p * 4 + (lane >> 4))] = own[p][q0 + q];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if constexpr (E::kPlain) put_rows<T, A, kAtOnce * kRows>(through, y, (t_own + q0) * kRows, (o0 + wo) * kRows);
            else finish_rows<E, A, kAtOnce * kRows>(through, y, e, (t_own + q0) * kRows, (o0 + wo) / kPerOutput<E> * kRows);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        return;
    }
    if constexpr (!E::kPlain) return;
    const int64_t t = t_own * kRows + (lane & 15), o = (o0 + wo) * kRows + (lane >> 4) * 4;
    float sx[kOwn];
    float4 sw[A];
#pragma unroll
    for (int q = 0; q < kOwn; ++q) sx[q] = token_scale(y, t + q * kRows);
#pragma unroll
    for (int p = 0; p < A; ++p) sw[p] = output_scales(y, o + p * kRows);
#pragma unroll
    for (int q = 0; q < kOwn; ++q)
#pragma unroll
        for (int p = 0; p < A; ++p) put4<T>(y, t + q * kRows, o + p * kRows, own[p][q], sx[q], sw[p]);
}

// Groups of 16 rows of the weight.
template <typename E>
int64_t pieces_of(const Scaled &y) {
    return cdiv(y.d_out, kRows) * kPerOutput<E>;
}

template <typename E>
int64_t tiles_of(const Scaled &y, int ot, int tt) {
    return cdiv(pieces_of<E>(y), ot) * cdiv(y.m, tt * kRows);
}

template <typename T, typename E, int OT, int TT, int WO, int WT, int G, int BUFS, bool BEHIND_FIRST = true>
void launch_tiles(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, const E &e, hipStream_t st) {
    const int o_tiles = (int)cdiv(pieces_of<E>(y), OT), t_tiles = (int)cdiv(y.m, TT * kRows);
    tile_kernel<T, E, OT, TT, WO, WT, G, BUFS, BEHIND_FIRST><<<dim3((unsigned)(o_tiles * t_tiles)), WO * WT * G * 64, 0, st>>>(W, X, deep, o_tiles, t_tiles, y, e);
}

template <typename T, typename E, int OP, int TP, int WAVES>
void launch_shared(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, const E &e, hipStream_t st) {
    const int64_t t_tiles = cdiv(y.m, TP * kRows), tiles = tiles_of<E>(y, OP, TP);
    shared_depth_kernel<T, E, OP, TP, WAVES><<<dim3((unsigned)tiles), WAVES * 64, 0, st>>>(W, X, deep, (int)t_tiles, y, e);
}

constexpr int64_t kUnits = 256;  // compute units

// Two pieces of outputs by two of tokens a workgroup, its wavefronts sharing the depth, where those are a round of the units: a long
// depth by 16 wavefronts, else by 8; twice the outputs by 4 wavefronts where there are more.  us (64 tokens 8192 -> 1024; 100 tokens
// 5120 -> 2048; 64 tokens 28672 -> 2048; 40 tokens 8192 -> 8192): by 16 7.0, 6.2, 21.2, 15.0, by 8 7.0, 6.2, 31.0, 14.0, twice the
// outputs 8.8, 7.1, 29.8, 13.8.
template <typename T, typename E>
void launch_pairs(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, const E &e, hipStream_t st) {
    const bool round = tiles_of<E>(y, 2, 2) <= kUnits;
    if (round && deep >= 96) launch_shared<T, E, 2, 2, 16>(W, X, deep, y, e, st);
    else if (round) launch_shared<T, E, 2, 2, 8>(W, X, deep, y, e, st);
    else launch_shared<T, E, 4, 2, 4>(W, X, deep, y, e, st);
}

// Which kernel: the largest tile that fills the chip.  A tile of 256 x 256 or 256 x 128 takes a compute unit for itself, so
// its last round has to be two thirds full, or one of many.  us (4096 tokens 8192 -> 28672; 2048 tokens 4096 -> 4096; 1024
// tokens 4096 -> 4096; 512 tokens 4096 -> 11008): 256 x 256 737, 60, 53, 53; 256 x 128 860, 43.1, 36, 34.8; 128 x 128 901,
// 44.0, 28, 35.4.
// Where 128 x 128 would be no more than one a unit: the smallest tile that is still at most one a unit, since the unit with most
// tiles is what all wait for, its depth shared by two or three groups of wavefronts, since one group alone keeps neither the
// matrix instructions nor the loads busy.  us of a round of each at a depth of 4096: 64 x 64 9, 96 x 48 10.9, 64 x 128 and 128 x 64
// 13.5, 96 x 96 14.8, 128 x 128 18 to 20, two rounds 17, 21, ...  Groups against one, 128 x 128: 700 tokens 4096 -> 4096 19.0 and
// 20.4, 200 tokens 2048 -> 13824 14.2 and 15.6.  One round against two of a smaller: 333 tokens 4099 -> 3001 96 x 48 12.9 (11.7 since its outputs
// pass through LDS), 64 x 128 14.8, 64 x 64 15.4; 150 tokens 4096 -> 11008 96 x 96 14.7, 64 x 64 19.4; 64 tokens 5120 -> 28672 128 x 64 25.7,
// 128 x 128 28.2; 400 tokens 8192 -> 5120 128 x 128 28.4, 64 x 64 34.8 (but 1000 tokens 2048 -> 2560 12.6 and 12.1).
// 64 x 64: a ring of 8 steps, since a unit's one workgroup has to have the weights' way from memory covered, and two groups for more than
// 128 tokens of 4096 inputs or more.  us with the codes, weights from memory (from the caches): 333 tokens 28672 -> 2048 one group 60.0 (55.1),
// two 59.7 (49.9), two with 4 steps 67.9 (50.5); 333 tokens 8192 -> 2560 23.7 (22.2), 23.4 (20.8), 25.6 (20.9); but 100 tokens 5120 -> 5120 18.1
// (15.3), 19.0 (14.4), 19.0 (14.3); 333 tokens 2048 -> 2048 10.9 (10.5), 11.2 (10.4), 10.9 (10.2).
// Fewer than 150 tiles of 64 x 64, and up to 32 tokens: wavefronts share the depth.  us without the codes, weights from the caches, shared and
// 64 x 64, 512 tokens of 4096: 128 tiles 7.6 and 9.3, 144 10.8 and 9.3, 152 10.8 and 9.4; of 1024: 4.8 and 6.0, 6.2 and 6.0, 6.2 and 6.0; 128
// tokens of 8192, weights from memory: 16.9 and 21.8, 26.5 and 21.6, 26.7 and 21.8 (pieces of two by two end at 128).
// Up to 16 tokens, us without the codes, weights from memory, 16 tokens of 4096 (of 13824):
//   pieces            256          304          320          512          520          752          768          832
//   two by 8       8.5 (22.4)   8.8 (22.7)   8.9 (22.8)   9.6 (25.4)  10.5 (29.7)  12.2 (33.2)  11.8 (33.5)  12.2 (34.9)
//   one by 8       7.5 (18.0)   8.2 (19.3)   8.2 (19.7)   9.7 (22.2)  11.0 (28.4)  11.9 (31.3)  11.5 (31.7)  15.5 (44.7)
//   two by 16      7.1 (17.0)   7.4 (17.5)   7.6 (17.7)   8.5 (21.5)  11.7 (32.9)  13.0 (37.2)  12.7 (37.1)  13.0 (38.1)
//   one by 16      6.1 (13.0)   8.8 (22.6)   8.9 (22.9)  10.2 (25.3)  11.7 (28.7)  12.5 (32.3)  12.3 (32.6)  14.8 (40.1)
// A round of the units is 256 workgroups, of small ones (8 wavefronts) three.
template <typename T, typename E>
int launch_product(const uint8_t *W, const uint8_t *X, int deep, const Scaled &y, const E &e, hipStream_t st) {
    auto fills = [](int64_t n) { return n >= 4 * kUnits || (n + kUnits / 3) / kUnits * kUnits >= n; };  // 171 .. 256, 427 .. 512, ...
    const int64_t pieces = pieces_of<E>(y);
    constexpr int kLeast = kPerOutput<E>;  // pieces of a workgroup at least
    if (tiles_of<E>(y, kLeast, 1) > INT32_MAX) return CMPQ_ESHAPE;
    if (y.m <= 16 && pieces >= 768) launch_shared<T, E, 2, 1, 8>(W, X, deep, y, e, st);
    else if (y.m <= 16 && pieces > 512) launch_shared<T, E, kLeast, 1, 8>(W, X, deep, y, e, st);
    else if (y.m <= 16 && pieces >= 320) launch_shared<T, E, 2, 1, 16>(W, X, deep, y, e, st);
    else if (y.m <= 16) launch_shared<T, E, kLeast, 1, 16>(W, X, deep, y, e, st);
    else if (y.m <= 32) launch_pairs<T, E>(W, X, deep, y, e, st);
    else if (fills(tiles_of<E>(y, 16, 16))) launch_tiles<T, E, 16, 16, 4, 2, 1, 4>(W, X, deep, y, e, st);
    else if (fills(tiles_of<E>(y, 16, 8))) launch_tiles<T, E, 16, 8, 4, 2, 1, 4>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 8, 8) > 2 * kUnits) launch_tiles<T, E, 8, 8, 2, 2, 1, 4, false>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 8, 8) > kUnits) launch_tiles<T, E, 8, 8, 2, 2, 1, 4>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 4, 4) < 150) launch_pairs<T, E>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 4, 4) <= kUnits && y.m > 128 && deep >= 64) launch_tiles<T, E, 4, 4, 2, 2, 2, 8>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 4, 4) <= kUnits) launch_tiles<T, E, 4, 4, 2, 2, 1, 8>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 6, 3) <= kUnits) launch_tiles<T, E, 6, 3, 3, 1, 3, 4>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 4, 8) <= kUnits) launch_tiles<T, E, 4, 8, 2, 2, 2, 4>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 8, 4) <= kUnits) launch_tiles<T, E, 8, 4, 2, 2, 2, 4>(W, X, deep, y, e, st);
    else if (tiles_of<E>(y, 6, 6) <= kUnits) launch_tiles<T, E, 6, 6, 3, 1, 3, 4>(W, X, deep, y, e, st);
    else launch_tiles<T, E, 8, 8, 2, 2, 2, 4>(W, X, deep, y, e, st);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

// Whether one token's product is better off with 8 wavefronts a workgroup than with 16.  Weights from memory, us with 8 and 16: 2048 -> 28672
// 13.2 and 16.0, 5120 -> 13824 15.9 and 18.0, 1000 -> 4096 4.7 and 4.5 (from the caches 4.1 and 4.5); but 2048 -> 4096 5.1 and 4.5, 4096 -> 4096 7.2
// and 5.7, -> 28672 22.6 and 21.8, 5120 -> 4096 8.0 and 6.9, -> 8192 10.9 and 11.2 (9.2 and 7.9).  Where workgroups are few, those of 8 lie two in
// a unit beside units without one; of up to 4096 inputs 16 bring all they need at once, and 8 half of more than 2048.
bool eight_wavefronts(const Scaled &y, int64_t d) {
    const int64_t pieces = cdiv(y.d_out, kRows);
    return d <= 1024 || (d <= 2048 && pieces > kUnits) || (d > 4096 && d <= 6144 && pieces > 2 * kUnits);
}

// Whether the tokens go in one launch.
template <typename E>
bool few_fit(const Scaled &y, int64_t d) {
    if (y.m == 1) return d <= 2 * kFewDepth;
    return y.m == 2 && (d <= kFewDepth || (!E::kGated && d <= 2 * kFewDepth && pieces_of<E>(y) <= 256));
}

template <typename TX, typename E>
void launch_few(const uint8_t *W, const void *X, int64_t d, int64_t ldx, const Scaled &y, const E &e, int y_dtype, int32_t *status,
                hipStream_t st) {
    const dim3 grid((unsigned)cdiv(y.d_out, kRows));
    const TX *x = static_cast<const TX *>(X);
    const int deep = (int)pieces_deep(d);
    const auto run = [&](auto tokens, auto chunks, auto waves) {
        few_tokens_kernel<TX, E, tokens(), chunks(), waves()><<<grid, waves() * 64, 0, st>>>(W, x, d, ldx, deep, y, e, y_dtype, status);
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    typedef std::integral_constant<int, 8> Eight;
    typedef std::integral_constant<int, 16> Sixteen;
    if (y.m == 2) {
        if (d <= kFewDepth) run(Two(), One(), Sixteen());
        else if constexpr (!E::kGated) run(Two(), Two(), Sixteen());
    } else if (!E::kGated && eight_wavefronts(y, d)) {
        if constexpr (!E::kGated) run(One(), One(), Eight());
    } else {
        if (d <= kFewDepth) run(One(), One(), Sixteen());
        else run(One(), Two(), Sixteen());
    }
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
bool gated_sizes_fit(int64_t d_in, int64_t d_out) { return d_in <= kMostDepth && d_out < (1 << 23); }

// What every form of the product is asked for.
struct Asked {
    const void *X;  // null: rows in 8 bits
    int dtype;
    int64_t d_in, ldx;
    const int8_t *x_codes, *codes;
    int y_dtype;
    int32_t *status;
};

// Codes the rows if they are not coded yet, then multiplies.  `y.sx` is filled in here.
template <typename E>
int run_product(const Asked &a, Scaled y, const E &e, const Work &w, hipStream_t st) {
    const uint8_t *cw = reinterpret_cast<const uint8_t *>(a.codes);
    if (a.X && few_fit<E>(y, a.d_in)) {
        if (a.dtype == CMPQ_F16) launch_few<_Float16>(cw, a.X, a.d_in, a.ldx, y, e, a.y_dtype, a.status, st);
        else if (a.dtype == CMPQ_BF16) launch_few<__bf16>(cw, a.X, a.d_in, a.ldx, y, e, a.y_dtype, a.status, st);
        else launch_few<float>(cw, a.X, a.d_in, a.ldx, y, e, a.y_dtype, a.status, st);
        CMPQ_LAUNCH_CHECK();
        return CMPQ_OK;
    }
    const uint8_t *cx = reinterpret_cast<const uint8_t *>(a.x_codes);
    if (a.X) {
        if (int rc = launch_code_rows_of(a.X, a.dtype, y.m, a.d_in, a.ldx, y.m, w.codes, w.scale, {1, 0}, a.status, st)) return rc;
        cx = reinterpret_cast<const uint8_t *>(w.codes);
        y.sx = w.scale;
    }
    const int deep = (int)pieces_deep(a.d_in);
    if constexpr (E::kPlain) {
        if (a.y_dtype == CMPQ_F16) return launch_product<_Float16>(cw, cx, deep, y, e, st);
        if (a.y_dtype == CMPQ_BF16) return launch_product<__bf16>(cw, cx, deep, y, e, st);
    }
    return launch_product<float>(cw, cx, deep, y, e, st);
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Whether four outputs next to each other may be written, and their scales read, at once.
bool fours(const void *Y, int y_dtype, int64_t ldy, const float *scale) {
    return ldy % 4 == 0 && reinterpret_cast<uintptr_t>(Y) % (4 * dtype_bytes(y_dtype)) == 0 && aligned16(scale);
}

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
    if (!W || !codes || !scale || !aligned16(codes)) return CMPQ_EINVAL;
    if (ldw < d_in || !sizes_fit(d_in, d_out)) return CMPQ_ESHAPE;
    return launch_code_rows_of(W, dtype, d_out, d_in, ldw, cdiv(d_out, kRows) * kRows, codes, scale, {1, 0}, status,
                            static_cast<hipStream_t>(stream));
}

extern "C" int64_t cmpq_int8_gated_rows(int64_t d_out) { return d_out < 0 || d_out >= (1 << 23) ? 0 : cdiv(d_out, kRows) * 2 * kRows; }

extern "C" int cmpq_int8_prepare_gated(const void *gate, const void *up, int dtype, int64_t d_out, int64_t d_in,
                                       int64_t ld_gate, int64_t ld_up, int8_t *codes, float *scale, int32_t *status,
                                       void *stream) {
    if (d_out < 0 || d_in < 0 || !serving_dtype(dtype)) return CMPQ_EINVAL;
    if (d_out == 0 || d_in == 0) return CMPQ_OK;
    if (!gate || !up || !codes || !scale || !aligned16(codes)) return CMPQ_EINVAL;
    if (ld_gate < d_in || ld_up < d_in || !gated_sizes_fit(d_in, d_out)) return CMPQ_ESHAPE;
    const int64_t rows = cdiv(d_out, kRows) * kRows;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int rc = launch_code_rows_of(gate, dtype, d_out, d_in, ld_gate, rows, codes, scale, {2, 0}, status, st)) return rc;
    return launch_code_rows_of(up, dtype, d_out, d_in, ld_up, rows, codes, scale, {2, 1}, status, st);
}

extern "C" int cmpq_int8_product(const void *X, int dtype, int64_t m, int64_t d_in, int64_t ldx, const int8_t *codes,
                                 const float *scale, int64_t d_out, void *Y, int y_dtype, int64_t ldy, void *ws,
                                 size_t ws_bytes, int32_t *status, void *stream) {
    if (m < 0 || d_in < 1 || d_out < 0 || !serving_dtype(dtype) || !serving_dtype(y_dtype)) return CMPQ_EINVAL;
    if (m == 0 || d_out == 0) return CMPQ_OK;
    if (!X || !codes || !scale || !Y || !aligned16(codes)) return CMPQ_EINVAL;
    if (ldx < d_in || ldy < d_out || m >= (1 << 24) || !sizes_fit(d_in, d_out)) return CMPQ_ESHAPE;
    const Work w = carve(ws, m, d_in);
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < w.bytes) return CMPQ_EWORKSPACE;
    const Scaled y = {nullptr, scale, Y, m, d_out, ldy, fours(Y, y_dtype, ldy, scale)};
    return run_product(Asked{X, dtype, d_in, ldx, nullptr, codes, y_dtype, status}, y, Plain(), w, static_cast<hipStream_t>(stream));
}

int cmpq_check_int8_product(const cmpq_int8_job *j) {
    if (!j || j->m < 0 || j->d_in < 1 || j->d_out < 0 || !serving_dtype(j->y_dtype) || !known_activation(j->activation)) return CMPQ_EINVAL;
    if (j->X && !serving_dtype(j->x_dtype)) return CMPQ_EINVAL;
    if ((j->bias || j->up_bias) && !serving_dtype(j->bias_dtype)) return CMPQ_EINVAL;
    if ((j->residual && !serving_dtype(j->r_dtype)) || (j->up_bias && !j->gated)) return CMPQ_EINVAL;
    if (j->m == 0 || j->d_out == 0) return CMPQ_OK;
    if (!j->codes || !j->scale || !j->Y || !aligned16(j->codes)) return CMPQ_EINVAL;
    if (!j->X && (!j->x_codes || !j->x_scale || !aligned16(j->x_codes))) return CMPQ_EINVAL;
    if ((j->X && j->ldx < j->d_in) || j->ldy < j->d_out || (j->residual && j->ldr < j->d_out)) return CMPQ_ESHAPE;
    if (j->m >= (1 << 24) || !(j->gated ? gated_sizes_fit : sizes_fit)(j->d_in, j->d_out)) return CMPQ_ESHAPE;
    return CMPQ_OK;
}

extern "C" int cmpq_int8_product_job(const cmpq_int8_job *j, void *ws, size_t ws_bytes, void *stream) {
    if (int rc = cmpq_check_int8_product(j)) return rc;
    if (j->m == 0 || j->d_out == 0) return CMPQ_OK;
    Work w = {};
    if (j->X) {
        w = carve(ws, j->m, j->d_in);
        if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < w.bytes) return CMPQ_EWORKSPACE;
    }
    const Scaled y = {j->X ? nullptr : j->x_scale, j->scale, j->Y, j->m, j->d_out, j->ldy, fours(j->Y, j->y_dtype, j->ldy, j->scale)};
    const Asked a = {j->X, j->x_dtype, j->d_in, j->ldx, j->x_codes, j->codes, j->y_dtype, j->status};
    hipStream_t st = static_cast<hipStream_t>(stream);
    Epilogue e;
    e.bias = j->bias, e.up_bias = j->up_bias, e.residual = j->residual, e.ldr = j->ldr;
    e.bias_dtype = j->bias_dtype, e.r_dtype = j->r_dtype, e.y_dtype = j->y_dtype, e.act = j->activation;
    if (j->gated) {
        GatedEpilogue g;
        static_cast<Epilogue &>(g) = e;
        return run_product(a, y, g, w, st);
    }
    if (!e.bias && !e.residual && e.act == CMPQ_ACT_NONE) return run_product(a, y, Plain(), w, st);
    return run_product(a, y, e, w, st);
}
