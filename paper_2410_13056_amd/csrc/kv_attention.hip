// Attention over the paged cache in 8 bits.
//
// The products are formed transposed, S^T = K Q^T and O^T = V^T P^T, with 16x16x32 FP16 matrix instructions: what the
// first leaves in a lane (4 tokens of one query row, twice) is what the second takes from it, so logits and weights
// never leave registers, and a lane's share of the running maximum and sum belongs to one query row.  A wavefront takes 32
// tokens (a unit) at a time; their codes are stored in the order of the instruction's operands, 16 bytes a lane and
// 1 KB a load, and become FP16 exactly: byte b under 0x64 is 1024 + b.  A page's key scale multiplies its
// logits and its value scale its weights, both in fp32.
#include "serving.h"

namespace {

typedef _Float16 Half2 __attribute__((ext_vector_type(2)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
typedef float Float4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 32;                  // tokens
constexpr int kWaves = 4;                  // wavefronts that share a part of a sequence
constexpr int kLeast = 8;                  // units of a part
constexpr int64_t kTarget = 1024;          // parts that fill the chip
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kSlack = 8.f;              // a row's logits pass its reference by a factor of at most 2^kSlack
constexpr float kRaise = 7.f;              // weights are held times 2^kRaise: at most 2^15 in FP16

struct Job {
    cmpq_kv_cache c;
    const int32_t *table, *lengths, *cu;
    int64_t ld_table, n_seq, n_rows, max_rows, max_length;
    cmpq_heads Q, O;
    int q_dtype, o_dtype, q_heads, group;
    float scale;
    int causal;
    int64_t window;
    cmpq_rotation rot;
    int32_t *status;
    float *part_o, *part_ml;   // [slots, columns, dims], [slots, columns, 2]
    int64_t slots;
};

// A sequence: its rows and tokens, cut to what the call allows.
struct Seq {
    int64_t row0;
    int rows, asked, length;   // `asked`: rows that the call names (the first `rows` of them are done)
    int first_unit, units;     // those that some row attends to
};

__device__ __forceinline__ Seq sequence(const Job &j, int64_t i, bool &bad) {
    Seq s;
    const int64_t a = j.cu[i], b = j.cu[i + 1];
    s.row0 = min(max(a, (int64_t)0), j.n_rows);
    const int64_t end = min(max(b, s.row0), j.n_rows);
    s.asked = (int)(end - s.row0);
    s.rows = (int)min((int64_t)s.asked, j.max_rows);
    const int64_t named = j.lengths[i];
    const int64_t length = min(max(named, (int64_t)0), min(j.max_length, j.ld_table * j.c.page));
    bad |= a != s.row0 || b != end || s.rows != s.asked || length != named;
    s.length = (int)length;
    const int64_t low = j.window > 0 ? max((int64_t)0, length - s.asked - j.window + 1) : 0;
    s.first_unit = (int)(low / kUnit);
    s.units = max(0, (int)((length + kUnit - 1) / kUnit) - s.first_unit);
    return s;
}

// How the call's work is cut up: a tile is NC (row, query head of the group) pairs of a sequence, a part at most `step`
// units of it.  Every wavefront works this out for itself from the lengths, 64 sequences at a time.
struct Plan {
    int step;
};

template <int NC>
__device__ __forceinline__ int tiles_of(const Job &j, const Seq &s) {
    return (int)(((int64_t)s.rows * j.group + NC - 1) / NC);
}

template <int NC>
__device__ __forceinline__ Plan make_plan(const Job &j, bool look) {
    const int lane = threadIdx.x & 63;
    double total = 0;
    for (int64_t base = 0; base < j.n_seq; base += 64) {
        if (base + lane >= j.n_seq) continue;
        bool bad = false;
        const Seq s = sequence(j, base + lane, bad);
        if (bad && look && j.status) atomicOr(j.status, CMPQ_STATUS_RANGE);
        total += (double)s.units * tiles_of<NC>(j, s);
    }
    total = wave_sum_f64(total);
    const double all = __shfl(total, 0) * j.c.kv_heads;
    Plan p;
    p.step = max(kLeast, (int)ceil(all / (double)kTarget));
    return p;
}

__device__ __forceinline__ int parts_of(const Plan &p, const Seq &s) { return max(1, (s.units + p.step - 1) / p.step); }

// Sequence that holds slot `x`, and the slots of those before it; seq < 0: there is no such slot.
struct Place {
    int64_t seq, before;
};

template <int NC>
__device__ __forceinline__ Place place_of(const Job &j, const Plan &p, int64_t x) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int64_t base = 0; base < j.n_seq; base += 64) {
        uint32_t n = 0;
        if (base + lane < j.n_seq) {
            bool bad = false;
            const Seq s = sequence(j, base + lane, bad);
            n = (uint32_t)(parts_of(p, s) * tiles_of<NC>(j, s) * j.c.kv_heads);
        }
        const uint32_t incl = wave_scan_incl_u32(n);
        const uint64_t past = __ballot(before + incl > x);
        if (past) {
            const int l = __builtin_ctzll(past);
            return {base + l, before + (int64_t)(__shfl(incl, l) - __shfl(n, l))};
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
    return {-1, 0};
}

// Eight codes (bytes code + 128) as FP16.
__device__ __forceinline__ Half8 halves(uint32_t a, uint32_t b) {
    union {
        uint32_t w[4];
        Half2 h[4];
        Half8 v;
    } u;
    u.w[0] = __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u);
    u.w[1] = __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u);
    u.w[2] = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
    u.w[3] = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
    const Half2 off = {(_Float16)1152.f, (_Float16)1152.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) u.h[i] -= off;
    return u.v;
}

// Largest over the four lanes that hold the same query row (lanes 16 apart), in all of them.
__device__ __forceinline__ float rows_max(float v) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float v) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const uint32_t w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ void put(const Job &j, int64_t row, int head, int d, float v) {
    const int64_t at = row * j.O.row_stride + head * j.O.head_stride + d;
    if (j.o_dtype == CMPQ_F16) static_cast<_Float16 *>(j.O.ptr)[at] = (_Float16)v;
    else static_cast<__bf16 *>(j.O.ptr)[at] = (__bf16)v;
}

// A query row's dims as the matrix instruction takes them, times 2^-e so that the largest lies in 1..2: lane
// 16 g + n has dims 32 c + 8 g .. + 7 of row n.  Returns 2^e.
template <int C>
__device__ __forceinline__ float load_query(const Job &j, int64_t row, int head, int64_t pos, Half8 (&q)[C]) {
    const int lane = threadIdx.x & 63, dim = j.c.head_dim;
    float x[C][8], most = 0.f;
    with_dtype(j.q_dtype, [&](auto like) {
        using T = decltype(like);
        const T *p = static_cast<const T *>(j.Q.ptr) + row * j.Q.row_stride + head * j.Q.head_stride;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = c * 32 + (lane >> 4) * 8 + i;
                x[c][i] = d < dim ? turned(p, d, j.rot, pos) : 0.f;
            }
    });
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[c][i]));
    most = rows_max(most);
    const int e = most > 0.f && most < INFINITY ? ilogbf(most) : 0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) q[c][i] = (_Float16)ldexpf(x[c][i], -e);
    return ldexpf(1.f, e);
}

// C: 32 dims each of a head.  Tiles of 16 columns, one (row, query head) pair each; the wavefronts take the
// part's units in turn and are added up through LDS.
template <int C>
__global__ __launch_bounds__(kWaves * 64) void attend_kernel(Job j) {
    constexpr int NC = 16, DP = C * 32, kPad = DP + 4;
    __shared__ float red[kWaves * NC * kPad];
    __shared__ float ml[kWaves][NC][2];
    const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, g = lane >> 4;
    const Plan plan = make_plan<NC>(j, blockIdx.x == 0 && wave == 0);
    const Place place = place_of<NC>(j, plan, blockIdx.x);
    if (place.seq < 0) return;
    bool bad = false;
    const Seq s = sequence(j, place.seq, bad);
    const int tiles = tiles_of<NC>(j, s), parts = parts_of(plan, s);
    const int64_t x = blockIdx.x - place.before;
    const int tile = (int)(x % tiles), head = (int)(x / tiles % j.c.kv_heads), part = (int)(x / tiles / j.c.kv_heads);

    // this lane's query row
    const int col = min(tile * NC + n, s.rows * j.group - 1);
    const int row = col / j.group, qh = head * j.group + col % j.group;
    const int64_t pos = (int64_t)s.length - s.asked + row;
    int64_t at = max(pos, (int64_t)0);
    if (j.rot.cos && at >= j.rot.positions) {
        at = j.rot.positions - 1;
        if (j.status) atomicOr(j.status, CMPQ_STATUS_RANGE);
    }
    Half8 q[C];
    const float factor = load_query<C>(j, s.row0 + row, qh, at, q) * j.scale * kLog2e;
    const int hi = (int)(j.causal ? min((int64_t)s.length, pos + 1) : (int64_t)s.length);  // tokens lo .. hi-1
    const int lo = j.window > 0 ? (int)max((int64_t)0, pos - j.window + 1) : 0;
    // bounds over the tile's rows: rows grow with the column
    const int all_hi = __builtin_amdgcn_readlane(hi, 0), all_lo = __builtin_amdgcn_readlane(lo, 15);

    Float4 o[2 * C];
#pragma unroll
    for (int d = 0; d < 2 * C; ++d) o[d] = Float4{0.f, 0.f, 0.f, 0.f};
    float m = -3.4e38f, sum = 0.f, unit_scale = 0.f;  // reference, this lane's share of the sum, value scale of o

    const int u0 = s.first_unit + part * plan.step, u1 = min(u0 + plan.step, s.first_unit + s.units);
    const int64_t page_bytes = (int64_t)j.c.page * DP;
    for (int base = u0 + wave; base < u1; base += kWaves * 64) {
        // pages and scales of 64 units of this wavefront at once
        const int mine = base + lane * kWaves;
        int id = -1, in_page = 0;
        float ks = 0.f, vs = 0.f;
        if (mine < u1) {
            const int token = mine * kUnit;
            id = j.table[place.seq * j.ld_table + token / j.c.page];
            in_page = token % j.c.page / kUnit;
            if (id < 0 || id >= j.c.n_pages) {
                id = -1;
                if (j.status) atomicOr(j.status, CMPQ_STATUS_RANGE);
            } else {
                ks = j.c.k_scale[(int64_t)id * j.c.kv_heads + head];
                vs = j.c.v_scale[(int64_t)id * j.c.kv_heads + head];
            }
        }
        const int count = min(64, (u1 - base + kWaves - 1) / kWaves);
        for (int i = 0; i < count; ++i) {
            const int page = __builtin_amdgcn_readlane(id, i);
            if (page < 0) continue;
            const float kscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), i));
            const float vscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), i));
            const int64_t off = ((int64_t)page * j.c.kv_heads + head) * page_bytes +
                                (int64_t)__builtin_amdgcn_readlane(in_page, i) * (kUnit * DP) + lane * 16;
            uint4 kc[C], vc[C];
#pragma unroll
            for (int c = 0; c < C; ++c) kc[c] = *reinterpret_cast<const uint4 *>(j.c.k_codes + off + c * 1024);
#pragma unroll
            for (int c = 0; c < C; ++c) vc[c] = *reinterpret_cast<const uint4 *>(j.c.v_codes + off + c * 1024);
            Float4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                s0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(kc[c].x, kc[c].y), q[c], s0, 0, 0, 0);
                s1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(kc[c].z, kc[c].w), q[c], s1, 0, 0, 0);
            }
            float l[8];
            const float f = factor * kscale;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                l[r] = s0[r] * f;
                l[4 + r] = s1[r] * f;
            }
            const int t0 = (base + i * kWaves) * kUnit;
            if (t0 < all_lo || t0 + kUnit > all_hi) {
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int t = t0 + (r >> 2) * 16 + g * 4 + (r & 3);
                    if (t < lo || t >= hi) l[r] = -INFINITY;
                }
            }
            float top = l[0];
#pragma unroll
            for (int r = 1; r < 8; ++r) top = fmaxf(top, l[r]);
            if (__ballot(top > m + kSlack) || vscale > unit_scale) {
                top = rows_max(top);  // a row's reference moves by its own logits alone
                const float next = top > m + kSlack ? top : m, keep = __builtin_amdgcn_exp2f(m - next);
                const float u = fmaxf(unit_scale, vscale), turn = keep * (unit_scale / u);
                sum *= keep;
#pragma unroll
                for (int d = 0; d < 2 * C; ++d) o[d] *= turn;
                m = next;
                unit_scale = u;
            }
            const float ratio = vscale / unit_scale, base_m = m - kRaise;
            Half8 p;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const float w = __builtin_amdgcn_exp2f(l[r] - base_m);
                sum += w;
                p[r] = (_Float16)(w * ratio);
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                o[2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(vc[c].x, vc[c].y), p, o[2 * c], 0, 0, 0);
                o[2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(vc[c].z, vc[c].w), p, o[2 * c + 1], 0, 0, 0);
            }
        }
    }

    // the wavefronts' shares: to one reference, then added in order
    sum = rows_sum(sum);
    if (g == 0) {
        ml[wave][n][0] = m;
        ml[wave][n][1] = sum;
    }
    __syncthreads();
    float top = ml[0][n][0], total = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml[w][n][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += ml[w][n][1] * __builtin_amdgcn_exp2f(ml[w][n][0] - top);
    const float mine = __builtin_amdgcn_exp2f(m - top) * unit_scale;
#pragma unroll
    for (int d = 0; d < 2 * C; ++d)
        *reinterpret_cast<Float4 *>(&red[(wave * NC + n) * kPad + d * 16 + g * 4]) = o[d] * mine;
    if (parts > 1 && wave == 0 && g == 0) {
        j.part_ml[(blockIdx.x * (int64_t)NC + n) * 2] = top;
        j.part_ml[(blockIdx.x * (int64_t)NC + n) * 2 + 1] = total;
    }
    __syncthreads();
    if (wave == 0 && g == 0) ml[0][n][1] = total;
    __syncthreads();
    for (int e = threadIdx.x; e < NC * DP; e += kWaves * 64) {
        const int c = e / DP, d = e % DP;
        float v = red[c * kPad + d];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += red[(w * NC + c) * kPad + d];
        if (parts > 1) {
            j.part_o[(blockIdx.x * (int64_t)NC + c) * DP + d] = v;
        } else if (tile * NC + c < s.rows * j.group && d < j.c.head_dim) {
            const int k = tile * NC + c;
            const float t = ml[0][c][1];
            put(j, s.row0 + k / j.group, head * j.group + k % j.group, d, t == 0.f ? 0.f : v / t);
        }
    }
}

// Rows whose sequence was cut into several parts: one wavefront a row and query head.
template <int C>
__global__ __launch_bounds__(256) void join_kernel(Job j) {
    constexpr int NC = 16, DP = C * 32;
    const int lane = threadIdx.x & 63;
    const int64_t x = (int64_t)blockIdx.x * 4 + wave_index();
    const int64_t row = x / j.q_heads;
    const int qh = (int)(x % j.q_heads);
    if (row >= j.n_rows) return;
    const Plan plan = make_plan<NC>(j, false);
    // the row's sequence and the slots before it
    int64_t before = 0;
    for (int64_t base = 0; base < j.n_seq; base += 64) {
        uint32_t n = 0;
        Seq s = {};
        if (base + lane < j.n_seq) {
            bool bad = false;
            s = sequence(j, base + lane, bad);
            n = (uint32_t)(parts_of(plan, s) * tiles_of<NC>(j, s) * j.c.kv_heads);
        }
        const uint32_t incl = wave_scan_incl_u32(n);
        const uint64_t holds = __ballot(s.rows > 0 && row >= s.row0 && row < s.row0 + s.rows);
        if (holds) {
            const int l = __builtin_ctzll(holds);
            bool bad = false;
            s = sequence(j, base + l, bad);
            before += (int64_t)(__shfl(incl, l) - __shfl(n, l));
            const int parts = parts_of(plan, s), tiles = tiles_of<NC>(j, s);
            if (parts == 1) return;
            const int col = (int)(row - s.row0) * j.group + qh % j.group, head = qh / j.group;
            const int64_t slot0 = before + head * tiles + col / NC, step = (int64_t)tiles * j.c.kv_heads;
            if (slot0 + (parts - 1) * step >= j.slots) return;  // rows named twice: there is no room for their parts
            float top = -3.4e38f;
            for (int p = lane; p < parts; p += 64) top = fmaxf(top, j.part_ml[((slot0 + p * step) * NC + col % NC) * 2]);
#pragma unroll
            for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
            float total = 0.f, acc[(DP + 63) / 64] = {};
#pragma unroll 4
            for (int p = 0; p < parts; ++p) {
                const int64_t at = (slot0 + p * step) * NC + col % NC;
                const float w = __builtin_amdgcn_exp2f(j.part_ml[at * 2] - top);
                total += w * j.part_ml[at * 2 + 1];
#pragma unroll
                for (int k = 0; k < (DP + 63) / 64; ++k)
                    if (k * 64 + lane < DP) acc[k] += w * j.part_o[at * DP + k * 64 + lane];
            }
#pragma unroll
            for (int k = 0; k < (DP + 63) / 64; ++k)
                if (k * 64 + lane < j.c.head_dim) put(j, row, qh, k * 64 + lane, total == 0.f ? 0.f : acc[k] / total);
            return;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
}

// Slots of a call: parts filled to the full, and one more a tile and head.
int64_t tiles_bound(const cmpq_kv_attention_job *a, int nc) {
    const int64_t group = a->q_heads / a->cache.kv_heads;
    const int64_t by_rows = a->n_rows * group / nc + a->n_seq, by_most = a->n_seq * cdiv(a->max_rows * group, nc);
    return by_rows < by_most ? by_rows : by_most;
}
int64_t slots_bound(const cmpq_kv_attention_job *a, int nc) {
    const int64_t tiles = tiles_bound(a, nc) * a->cache.kv_heads, parts = cdiv(cdiv(a->max_length, kUnit) + 1, kLeast);
    return tiles * (parts > 1 ? parts : 1) < tiles + kTarget ? tiles * (parts > 1 ? parts : 1) : tiles + kTarget;
}
bool may_split(const cmpq_kv_attention_job *a) { return cdiv(a->max_length, kUnit) > kLeast; }

int check_job(const cmpq_kv_attention_job *a) {
    if (!a) return CMPQ_EINVAL;
    if (int rc = check_cache(a->cache)) return rc;
    if (a->n_seq < 0 || a->n_rows < 0 || a->max_rows < 0 || a->max_length < 0 || a->ld_table < 0 || a->window < 0)
        return CMPQ_EINVAL;
    if (!serving_dtype(a->q_dtype) || (a->o_dtype != CMPQ_F16 && a->o_dtype != CMPQ_BF16)) return CMPQ_EINVAL;
    if (a->q_heads < 1 || a->q_heads % a->cache.kv_heads) return CMPQ_EINVAL;
    if (a->n_seq > INT32_MAX || a->n_rows > INT32_MAX || a->max_length > INT32_MAX - kUnit || a->q_heads > 65535 ||
        a->ld_table > INT32_MAX || a->max_rows > INT32_MAX || a->n_rows * a->q_heads > ((int64_t)1 << 33))
        return CMPQ_ESHAPE;
    return check_rotation(&a->rotation, a->cache.head_dim);
}

template <int C>
void launch(const Job &j, int64_t slots, bool split, hipStream_t st) {
    attend_kernel<C><<<dim3((unsigned)slots), kWaves * 64, 0, st>>>(j);
    if (split) join_kernel<C><<<dim3((unsigned)cdiv(j.n_rows * j.q_heads, 4)), 256, 0, st>>>(j);
}

}  // namespace

extern "C" size_t cmpq_kv_attention_workspace(const cmpq_kv_attention_job *a) {
    if (!a || a->cache.kv_heads < 1 || a->q_heads < 1 || a->n_seq < 0 || a->n_rows < 0 || a->max_rows < 0 ||
        a->max_length < 0 || !cmpq_kv_page_bytes(a->cache.head_dim, a->cache.page))
        return 0;
    WsCarver w(nullptr);
    const int64_t slots = may_split(a) ? slots_bound(a, 16) : 0, dp = cdiv(a->cache.head_dim, 32) * 32;
    w.take<float>((size_t)(slots * 16 * dp));
    w.take<float>((size_t)(slots * 16 * 2));
    return w.need() > 256 ? w.need() : 256;
}

extern "C" int cmpq_kv_attention(const cmpq_kv_attention_job *a, void *ws, size_t ws_bytes, void *stream) {
    if (int rc = check_job(a)) return rc;
    if (a->n_seq == 0 || a->n_rows == 0 || a->max_rows == 0) return CMPQ_OK;
    if (!a->page_table || !a->lengths || !a->cu_rows || !a->Q.ptr || !a->O.ptr) return CMPQ_EINVAL;
    const int64_t slots = slots_bound(a, 16), dp = cdiv(a->cache.head_dim, 32) * 32;
    if (slots > INT32_MAX) return CMPQ_ESHAPE;
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < cmpq_kv_attention_workspace(a)) return CMPQ_EWORKSPACE;
    const bool split = may_split(a);
    WsCarver w(ws);
    Job j = {};
    j.c = a->cache;
    j.table = a->page_table, j.lengths = a->lengths, j.cu = a->cu_rows;
    j.ld_table = a->ld_table, j.n_seq = a->n_seq, j.n_rows = a->n_rows, j.max_rows = a->max_rows, j.max_length = a->max_length;
    j.Q = a->Q, j.O = a->O, j.q_dtype = a->q_dtype, j.o_dtype = a->o_dtype, j.q_heads = a->q_heads;
    j.group = a->q_heads / a->cache.kv_heads;
    j.scale = a->softmax_scale, j.causal = a->causal, j.window = a->window, j.rot = a->rotation, j.status = a->status;
    j.slots = slots;
    j.part_o = w.take<float>((size_t)(split ? slots * 16 * dp : 0));
    j.part_ml = w.take<float>((size_t)(split ? slots * 16 * 2 : 0));
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (dp / 32) {
        case 1: launch<1>(j, slots, split, st); break;
        case 2: launch<2>(j, slots, split, st); break;
        case 3: launch<3>(j, slots, split, st); break;
        case 4: launch<4>(j, slots, split, st); break;
        case 5: launch<5>(j, slots, split, st); break;
        case 6: launch<6>(j, slots, split, st); break;
        case 7: launch<7>(j, slots, split, st); break;
        default: launch<8>(j, slots, split, st); break;
    }
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
