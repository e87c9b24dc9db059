// Attention over the paged cache in 8 bits.
//
// The products are formed transposed, S^T = K Q^T and O^T = V^T P^T: what the first matrix instruction leaves in a lane (4
// tokens of one query row, twice) is what the second takes from it, so logits and weights never leave registers, and a
// lane's share of the running maximum and sum belongs to one query row.  A wavefront takes 32 tokens (a unit) at a time; their
// codes are stored in the order of the instructions' operands, 16 bytes a lane and 1 KB a load.  A page's key scale
// multiplies its logits, its value scale goes into its weights' exponent.
//
// A row has two references, both running maxima over the tokens that it sees: m of its logits, against which the weights' sum
// is held, and m + d of its logits plus the logarithms of their value scales, against which its output is.  So the
// weights that a matrix instruction takes are near the top of FP16 where they matter for the output, whatever the scales
// of other pages.  A reference moves only when it is passed by a factor of 2^8, so that sums and outputs are rarely
// multiplied again; m cancels in the quotient, 2^d multiplies it at the end.
//
// Two kernels.  For few rows (attend_kernel) the cache's bytes are what counts: the wavefronts of a workgroup share the
// tokens and read codes straight from memory.  For many rows (attend_rows_kernel) multiplications and exponentials
// count: the wavefronts share the rows, and a workgroup's codes go through LDS.  A long sequence's units are cut into parts,
// which a second launch joins.
//
// Roundings: queries to 16 bits fixed point (fixed_query), their products with codes exact; weights to FP16 for the matrix
// instruction (their sum is taken before, in fp32); the output once to its type.  All else is fp32.
#include "serving.h"

namespace {

typedef _Float16 Half2 __attribute__((ext_vector_type(2)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef int32_t Int4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 32;                  // tokens
constexpr int kWaves = 4;                  // wavefronts of a workgroup
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -3.4e38f;        // a row's reference before its first token
constexpr float kSlack = 8.f;              // a row's logits pass its reference by a factor of at most 2^kSlack
constexpr float kRaise = 7.f;              // weights are held times 2^kRaise: at most 2^15 in FP16
constexpr float kMostBelow = 100.f;        // value scales further below 2^d count as 2^(d - kMostBelow)

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
    float *part_o, *part_ml;   // [kept, columns, dims], [kept, columns, 3]: outputs; m, d, sums
    int64_t kept;              // parts that there is room for
    int target, least;         // workgroups that fill the chip, units of a part at least
    int most_parts;            // of a sequence, by the host's bounds: the grid and the kept parts have room for so many
    int64_t least_cols, most_cols;  // sequences of that many (row, query head of the group) pairs are this kernel's
};

// A sequence: its rows and tokens, cut to what the call allows.
struct Seq {
    int64_t row0, at0;         // first row, and its position
    int rows, length;          // rows that are done of those that the call names
    int first_unit, units;     // those that some row attends to
};

__device__ __forceinline__ Seq sequence(const Job &j, int64_t i, bool &bad) {
    Seq s;
    const int64_t a = j.cu[i], b = j.cu[i + 1];
    s.row0 = min(max(a, (int64_t)0), j.n_rows);
    const int64_t end = min(max(b, s.row0), j.n_rows);
    const int64_t asked = end - s.row0, named = j.lengths[i], all = max(named, (int64_t)0);
    s.rows = (int)min(asked, j.max_rows);
    const int64_t length = min(all, min(j.max_length, j.ld_table * j.c.page));
    bad |= a != s.row0 || b != end || s.rows != asked || length != named;
    s.length = (int)length;
    s.at0 = all - asked;       // rows stay at their positions where tokens are left out
    const int64_t low = j.window > 0 ? max((int64_t)0, s.at0 - j.window + 1) : 0;
    s.first_unit = (int)(low / kUnit);
    s.units = max(0, (int)((length + kUnit - 1) / kUnit) - s.first_unit);
    return s;
}

// How the call's work is cut up: a tile is NC (row, query head of the group) pairs of a sequence, its units go in equal
// parts of at most `step`.  Every wavefront works this out for itself from the lengths, 64 sequences at a time.
struct Plan {
    int step, most_parts;
};

template <int NC>
__device__ __forceinline__ int tiles_of(const Job &j, const Seq &s) {
    const int64_t cols = (int64_t)s.rows * j.group;
    return cols < j.least_cols || cols > j.most_cols ? 0 : (int)((cols + NC - 1) / NC);
}

template <int NC>
__device__ __forceinline__ Plan make_plan(const Job &j, bool look) {
    const int lane = threadIdx.x & 63;
    if (j.kept == 0 && !look) return {1 << 30, 1};
    double total = 0, pieces = 0;
    for (int64_t base = 0; base < j.n_seq; base += 64) {
        if (base + lane >= j.n_seq) continue;
        bool bad = false;
        const Seq s = sequence(j, base + lane, bad);
        if (bad && look && j.status) atomicOr(j.status, CMPQ_STATUS_RANGE);
        total += (double)s.units * tiles_of<NC>(j, s);
        pieces += (double)tiles_of<NC>(j, s);
    }
    // a sequence's parts are rounded up: up to one workgroup a piece more than its share
    const double all = __shfl(wave_sum_f64(total), 0) * j.c.kv_heads, odd = __shfl(wave_sum_f64(pieces), 0) * j.c.kv_heads;
    Plan p;
    p.step = __builtin_amdgcn_readfirstlane(max(j.least, (int)ceil(all / max((double)j.target - odd, 0.5 * j.target))));
    if (j.kept == 0) p.step = 1 << 30;
    p.most_parts = j.most_parts;
    return p;
}

// A sequence that names more rows than `max_rows` may have more units in a window than the host counts with.
__device__ __forceinline__ int parts_of(const Plan &p, const Seq &s) {
    return min(max(1, (s.units + p.step - 1) / p.step), p.most_parts);
}

// A sequence's workgroups: those of the sequences before it, and how many of theirs leave parts to be joined (at most
// 2 target in all: a sequence of more than `step` units has at most 2 units / step parts).
struct Place {
    int64_t seq, before, kept_before;
};

// The sequence `wanted`, or that `is` tells apart, given its data and the workgroups up to and with it; seq < 0: none.
template <int NC, typename F>
__device__ __forceinline__ Place place_of(const Job &j, const Plan &p, F is, int64_t wanted = -1) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0, kept = 0;
    for (int64_t base = 0; base < j.n_seq; base += 64) {
        uint32_t n = 0, k = 0;
        Seq s = {};
        if (base + lane < j.n_seq) {
            bool bad = false;
            s = sequence(j, base + lane, bad);
            const int parts = parts_of(p, s);
            n = (uint32_t)(parts * tiles_of<NC>(j, s) * j.c.kv_heads);
            k = parts > 1 ? n : 0;
        }
        const uint32_t incl = wave_scan_incl_u32(n), kept_incl = wave_scan_incl_u32(k);
        const uint64_t found = __ballot(is(s, before + incl) || base + lane == wanted);
        if (found) {
            const int l = __builtin_ctzll(found);
            return {base + l, before + (uint32_t)__builtin_amdgcn_readlane((int)(incl - n), l),
                    kept + (uint32_t)__builtin_amdgcn_readlane((int)(kept_incl - k), l)};
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
        kept += (uint32_t)__builtin_amdgcn_readlane((int)kept_incl, 63);
    }
    return {-1, 0, 0};
}

// A workgroup's share: a tile of a sequence for a head, a part of its units; `slot`: where the part is kept.
struct Share {
    Seq s;
    int64_t seq, slot;
    int tile, head, parts, u0, u1;  // units u0 .. u1-1
};

template <int NC>
__device__ __forceinline__ bool share_of(const Job &j, const Plan &plan, int64_t x, Share &w) {
    const Place place = place_of<NC>(j, plan, [&](const Seq &, int64_t upto) { return upto > x; });
    if (place.seq < 0) return false;
    bool bad = false;
    w.seq = place.seq;
    w.s = sequence(j, place.seq, bad);
    w.parts = parts_of(plan, w.s);
    const int tiles = tiles_of<NC>(j, w.s);
    x -= place.before;
    w.slot = place.kept_before + x;
    w.tile = (int)(x % tiles);
    w.head = (int)(x / tiles % j.c.kv_heads);
    const int64_t part = x / tiles / j.c.kv_heads;
    w.u0 = w.s.first_unit + (int)(w.s.units * part / w.parts);
    w.u1 = w.s.first_unit + (int)(w.s.units * (part + 1) / w.parts);
    return w.parts == 1 || w.slot < j.kept;  // rows named twice: there is no room for their parts
}

// Eight codes (bytes code + 128) as FP16, exactly: byte b under 0x64 is 1024 + b.
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

// Over the four lanes that hold the same query row (lanes 16 apart), in all of them.
template <typename F>
__device__ __forceinline__ float over_row(float v, F both) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = both(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return both(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_max(float v) {
    return over_row(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float row_sum(float v) {
    return over_row(v, [](float a, float b) { return a + b; });
}

// Four dims next to each other of an output row.
__device__ __forceinline__ void put4(const Job &j, int64_t row, int head, int d, const Float4 &v) {
    const int64_t at = row * j.O.row_stride + head * j.O.head_stride + d;
    auto put = [&](auto like) {
        using T = decltype(like);
        typedef T T4 __attribute__((ext_vector_type(4)));
        typedef T4 Any __attribute__((aligned(sizeof(T))));
        T *p = static_cast<T *>(j.O.ptr) + at;
        if (d + 4 <= j.c.head_dim) {
            *reinterpret_cast<Any *>(p) = T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (d + r < j.c.head_dim) p[r] = (T)v[r];
        }
    };
    if (j.o_dtype == CMPQ_F16) put(_Float16());
    else put(__bf16());
}

// One column of a tile: a query row and head, and the tokens lo .. hi-1 that it sees.  Columns past the last repeat it.
struct Column {
    int64_t row, at;  // row of Q, row of the rotation's tables
    int head, lo, hi;
};

__device__ __forceinline__ Column column(const Job &j, const Seq &s, int kv_head, int index) {
    const int col = min(index, s.rows * j.group - 1);
    Column c;
    c.row = col / j.group;
    c.head = kv_head * j.group + col % j.group;
    const int64_t pos = s.at0 + c.row;
    c.row += s.row0;
    c.at = max(pos, (int64_t)0);
    if (j.rot.cos && c.at >= j.rot.positions) {
        c.at = j.rot.positions - 1;
        if (j.status) atomicOr(j.status, CMPQ_STATUS_RANGE);
    }
    c.hi = (int)(j.causal ? min((int64_t)s.length, pos + 1) : (int64_t)s.length);
    c.lo = j.window > 0 ? (int)max((int64_t)0, pos - j.window + 1) : 0;  // may be past the last token that is not left out
    return c;
}

// `count` columns of a head's queries from `index` on, turned, into LDS: rows of DP + 4 floats.  Threads first, first + step, ... take
// eight dims each; in a loop, since all of them at once take more registers than the kernels have left.
template <int C>
__device__ __forceinline__ void stage_queries(const Job &j, const Seq &s, int kv_head, int index, int count, float *to, int first,
                                              int step) {
    constexpr int DP = C * 32;
    const bool by_eight = turns_by_eight(j.rot);
#pragma unroll 1
    for (int e = first; e < count * (DP / 8); e += step) {
        const int n = e / (DP / 8), d = e % (DP / 8) * 8;
        const Column col = column(j, s, kv_head, index + n);
        float *row = to + n * (DP + 4) + d;
        with_dtype(j.q_dtype, [&](auto like) {
            using T = decltype(like);
            const T *p = static_cast<const T *>(j.Q.ptr) + col.row * j.Q.row_stride + col.head * j.Q.head_stride;
            if (by_eight && d + 8 <= j.c.head_dim) {
                float x[8];
                load_turned(p, d, j.rot, col.at * (j.rot.dims >> 1), x);
                *reinterpret_cast<Float4 *>(row) = Float4{x[0], x[1], x[2], x[3]};
                *reinterpret_cast<Float4 *>(row + 4) = Float4{x[4], x[5], x[6], x[7]};
            } else {
#pragma unroll 1
                for (int i = 0; i < 8; ++i) row[i] = d + i < j.c.head_dim ? turned(p, d + i, j.rot, col.at) : 0.f;
            }
        });
    }
}

// A staged row's dims in the lanes that hand them to the matrix instruction, scaled by a power of two so that the largest
// lies in 1..2: lane 16 g + n has dims 32 c + 8 g .. + 7 of row n.  Returns the exponent; `top` is that largest, NaN for
// a row that holds a NaN or an infinity.
template <int C>
__device__ __forceinline__ int take_query(const float *from, float (&x)[C][8], float &top) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    float most = 0.f, zero = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const Float4 *p = reinterpret_cast<const Float4 *>(from + (lane & 15) * (C * 32 + 4) + c * 32 + g * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[c][i] = p[i >> 2][i & 3];
            most = fmaxf(most, fabsf(x[c][i]));
            zero += x[c][i] * 0.f;  // NaN if one of them is no finite number
        }
    }
    most = row_max(most);
    const int e = most > 0.f && most < INFINITY ? ilogbf(most) : 0;
    top = ldexpf(most + row_sum(zero), -e);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = ldexpf(x[c][i], -e);
    return e;
}

// A staged row for the integer matrix instruction: 16 bits fixed point of the row's largest magnitude, 256 high + low, and
// what turns its products with codes into logits in base 2 (never below 0: the sign of softmax_scale goes into the
// row).  Keys then need no conversion, and two instructions of 64 dims do what two of 32 in FP16 would.  An element is
// off by at most 2^-16 of the row's largest, less than FP16 rounds the larger half of them by.
template <int C>
__device__ __forceinline__ float fixed_query(const float *from, float scale, bool seen, Int4 (&high)[(C + 1) / 2],
                                             Int4 (&low)[(C + 1) / 2]) {
    float v[C][8], top;
    const int e = take_query<C>(from, v, top);
    const float sign = scale < 0.f ? -1.f : 1.f, to = top > 0.f ? sign * 32639.f / top : 0.f;  // NaN: 0
#pragma unroll
    for (int c = 0; c < (C + 1) / 2 * 2; ++c) {
        uint32_t h[2] = {0, 0}, l[2] = {0, 0};
        if (c < C) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int q = (int)rintf(v[c < C ? c : 0][i] * to), up = (q + 128) >> 8;
                h[i >> 2] |= (uint32_t)(up & 255) << (8 * (i & 3));
                l[i >> 2] |= (uint32_t)((q - 256 * up) & 255) << (8 * (i & 3));
            }
        }
        high[c / 2][c % 2 * 2] = (int)h[0], high[c / 2][c % 2 * 2 + 1] = (int)h[1];
        low[c / 2][c % 2 * 2] = (int)l[0], low[c / 2][c % 2 * 2 + 1] = (int)l[1];
    }
    return seen ? ldexpf(top * (1.f / 32639.f) * (sign * scale * kLog2e), e) : 0.f;
}

// The page of a unit of a sequence, -1 if the table names none, and its scales.
struct PageOf {
    int id, in_page;
    float ks, vs, log_vs;
};

__device__ __forceinline__ PageOf page_of(const Job &j, int64_t seq, int head, int unit, int end) {
    PageOf p = {-1, 0, 0.f, 1.f, 0.f};
    if (unit >= end) return p;
    const int token = unit * kUnit, nth = token / j.c.page;
    p.id = j.table[seq * j.ld_table + nth];
    p.in_page = (token - nth * j.c.page) / kUnit;
    if (p.id < 0 || p.id >= j.c.n_pages) {
        p.id = -1;
        if (j.status) atomicOr(j.status, CMPQ_STATUS_RANGE);
    } else {
        p.ks = j.c.k_scale[(int64_t)p.id * j.c.kv_heads + head];
        p.vs = j.c.v_scale[(int64_t)p.id * j.c.kv_heads + head];
    }
    return p;
}
// The rest of it: apart, so that loads of the codes need not wait for the scales.
__device__ __forceinline__ void finish(PageOf &p) { p.log_vs = log2f(p.vs); }
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}

// A tile's running state of one column in a lane: the references m and d, this lane's share of the sum.
struct State {
    float m, d, sum;
};

// Logits that a unit's products s stand for (s times f), each row's largest; -infinity where the row does not see the token.
__device__ __forceinline__ float largest(const float (&s)[8], float f) {
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 8; ++r) top = fmaxf(top, s[r]);
    return top * f;
}

// What turns a row's products with a page's codes into logits: above 0, so that -infinity stays it; NaN stays NaN.
__device__ __forceinline__ float logit_factor(float of_row, float kscale) {
    const float f = of_row * kscale;
    return f < 0x1p-126f ? 0x1p-126f : f;
}

// Whether a unit's largest logit passes a reference of its row by more than the slack.
__device__ __forceinline__ bool passes(const State &st, float top, float log_vs) {
    return top - st.m > kSlack + fminf(0.f, st.d - log_vs);
}

// Moves the references that are passed, and what is held against them: by the row's own logits and pages alone, so results
// do not depend on the rows beside it.
template <int C, int NT>
__device__ __forceinline__ void move_up(State (&st)[NT], const float (&top)[NT], Float4 (&o)[NT][2 * C], float log_vs) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float now = row_max(top[t]), rise = now - st[t].m, below = st[t].d - log_vs;
        const bool up = rise > kSlack, out_up = rise - below > kSlack;
        st[t].sum *= up ? __builtin_amdgcn_exp2f(-rise) : 1.f;
        const float turn = out_up ? __builtin_amdgcn_exp2f(below - rise) : 1.f;
#pragma unroll
        for (int d = 0; d < 2 * C; ++d) o[t][d] *= turn;
        st[t].d = out_up ? log_vs + (up ? 0.f : rise) : st[t].d - (up ? rise : 0.f);
        st[t].m = up ? now : st[t].m;
    }
}

// The weights of a unit's 8 tokens in this lane to FP16, against m + d and with the unit's value scale; adds them to the sum,
// against m and without it.
__device__ __forceinline__ Half8 weigh(const float (&s)[8], float f, State &st, float log_vs) {
    const float below = fminf(st.d - log_vs, kMostBelow), base = st.m - kRaise + below;
    Half8 p;
    float w[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        w[r] = __builtin_amdgcn_exp2f(fmaf(s[r], f, -base));
        p[r] = (_Float16)w[r];
    }
    const float part = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    st.sum = fmaf(part, __builtin_amdgcn_exp2f(below), st.sum);
    return p;
}

// Output over sum, times 2^d, in two steps: 2^d may pass fp32's range where the result does not.
__device__ __forceinline__ Float4 quotient(const Float4 &o, float total, float d) {
    const float half = __builtin_amdgcn_exp2f(0.5f * d), by = total == 0.f ? 0.f : half / total;
    return o * by * half;
}

// What a part leaves of a column's output in the workspace, and beside it.
__device__ __forceinline__ void keep_part(const Job &j, int64_t slot, int nc, int col, int dims, int d, const Float4 &v) {
    *reinterpret_cast<Float4 *>(j.part_o + (slot * nc + col) * dims + d) = v;
}
__device__ __forceinline__ void keep_sum(const Job &j, int64_t slot, int nc, int col, float m, float d, float sum) {
    float *p = j.part_ml + (slot * nc + col) * 3;
    p[0] = m, p[1] = d, p[2] = sum;
}

// Few rows.  C: 32 dims each of a head.  Tiles of 16 NT columns, one (row, query head) pair each; the wavefronts take the
// part's units in turn and are added up through LDS.  Bound by the cache's bytes: 64 sequences of one row, 184 000 tokens,
// 8 heads of 128 dims in 76 us, 2 sequences of 172 000 tokens in 75 us (4.9 and 4.7 TB/s; a large copy reaches 4.8).  Where there
// is little to read, by what comes one after the other (lengths, pages, scales, queries, up to 4 units a wavefront, the join by
// barriers) on a part of the compute units: 11 us for 777 tokens of 32 heads, 32 workgroups.  Hence codes straight
// into registers a unit ahead, no barrier before the last unit, and the pages' numbers 64 at a time.
template <int C, int NT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : C * NT <= 4 ? 3 : C * NT <= 8 ? 2 : 1) void attend_kernel(Job j) {
    constexpr int NC = 16 * NT, DP = C * 32, kPad = DP + 4;
    __shared__ __align__(16) float red[4 * 16 * kPad];
    __shared__ float ml[WAVES][NC][3];
    const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, g = lane >> 4;
    const Plan plan = make_plan<NC>(j, blockIdx.x == 0 && wave == 0);
    Share w;
    if (!share_of<NC>(j, plan, blockIdx.x, w)) return;
    const Seq &s = w.s;
    const int tile = w.tile, head = w.head, parts = w.parts;

    static_assert(NT <= 4 && (WAVES == 4 || WAVES == 8), "room for the queries, shares of outputs");
    const int u0 = w.u0, u1 = w.u1;
    const int64_t page_bytes = (int64_t)j.c.page * DP;
    // pages of 64 units of this wavefront at once, and the codes of the unit to come: both before the queries, which take
    // their time as well
    int base = u0 + wave, count = 0;
    PageOf mine;
    uint4 kc[C], vc[C];
    auto load = [&](const uint8_t *from, int i, uint4 (&to)[C]) {
        const int k = min(i, count - 1);
        const int64_t off = ((int64_t)max(__builtin_amdgcn_readlane(mine.id, k), 0) * j.c.kv_heads + head) * page_bytes +
                            (int64_t)__builtin_amdgcn_readlane(mine.in_page, k) * (kUnit * DP) + lane * 16;
#pragma unroll
        for (int c = 0; c < C; ++c) to[c] = load16_stream(from + off + c * 1024);
    };
    auto begin = [&]() {
        mine = page_of(j, w.seq, head, base + lane * WAVES, u1);
        count = min(64, (u1 - base + WAVES - 1) / WAVES);
        load(j.c.k_codes, 0, kc);
        load(j.c.v_codes, 0, vc);
    };
    if (base < u1) begin();
    stage_queries<C>(j, s, head, tile * NC, NC, red, threadIdx.x, WAVES * 64);
    __syncthreads();
    Int4 qh[NT][(C + 1) / 2], ql[NT][(C + 1) / 2];
    float factor[NT];
    int lo[NT], hi[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const Column col = column(j, s, head, tile * NC + t * 16 + n);
        lo[t] = col.lo, hi[t] = col.hi;
        factor[t] = fixed_query<C>(red + t * 16 * kPad, j.scale, col.lo < col.hi, qh[t], ql[t]);
    }
    // bounds over the tile's columns: rows grow with the column
    const int all_hi = __builtin_amdgcn_readlane(hi[0], 0), all_lo = __builtin_amdgcn_readlane(lo[NT - 1], 15);

    Float4 o[NT][2 * C];
    State st[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        st[t] = {kLowest, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < 2 * C; ++d) o[t][d] = Float4{0.f, 0.f, 0.f, 0.f};
    }

    for (bool first = true; base < u1; base += WAVES * 64, first = false) {
        if (!first) begin();
        finish(mine);
        for (int i = 0; i < count; ++i) {
            const bool there = __builtin_amdgcn_readlane(mine.id, i) >= 0;
            const float kscale = lane_value(mine.ks, i), log_vs = lane_value(mine.log_vs, i);
            Int4 a[2][(C + 1) / 2];
#pragma unroll
            for (int c = 0; c < (C + 1) / 2; ++c) {
                const uint4 first = kc[2 * c], second = 2 * c + 1 < C ? kc[2 * c + 1 < C ? 2 * c + 1 : 0] : make_uint4(0, 0, 0, 0);
                constexpr uint32_t flip = 0x80808080u;  // code + 128 to the code's own byte
                a[0][c] = Int4{(int)(first.x ^ flip), (int)(first.y ^ flip), (int)(second.x ^ flip), (int)(second.y ^ flip)};
                a[1][c] = Int4{(int)(first.z ^ flip), (int)(first.w ^ flip), (int)(second.z ^ flip), (int)(second.w ^ flip)};
            }
            load(j.c.k_codes, i + 1, kc);
            float l[NT][8], top[NT];
            const int t0 = (base + i * WAVES) * kUnit;
            const bool edge = !there || t0 < all_lo || t0 + kUnit > all_hi;
            bool past = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                Int4 sum[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Int4 high = {}, low = {};
#pragma unroll
                    for (int c = 0; c < (C + 1) / 2; ++c) {
                        high = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[h][c], qh[t][c], high, 0, 0, 0);
                        low = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[h][c], ql[t][c], low, 0, 0, 0);
                    }
                    sum[h] = high * 256 + low;
                }
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int at = t0 + (r >> 2) * 16 + g * 4 + (r & 3);
                    l[t][r] = (float)sum[r >> 2][r & 3];
                    if (edge && (!there || at < lo[t] || at >= hi[t])) l[t][r] = -INFINITY;
                }
                top[t] = largest(l[t], logit_factor(factor[t], kscale));
                past |= passes(st[t], top[t], log_vs);
            }
            if (__ballot(past)) move_up<C, NT>(st, top, o, log_vs);
            Half8 p[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) p[t] = weigh(l[t], logit_factor(factor[t], kscale), st[t], log_vs);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const Half8 v0 = halves(vc[c].x, vc[c].y), v1 = halves(vc[c].z, vc[c].w);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    o[t][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[t], o[t][2 * c], 0, 0, 0);
                    o[t][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[t], o[t][2 * c + 1], 0, 0, 0);
                }
            }
            load(j.c.v_codes, i + 1, vc);
        }
    }

    // the wavefronts' shares: to one reference, then added in order, 16 columns at a time
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        st[t].sum = row_sum(st[t].sum);
        if (g == 0) {
            ml[wave][t * 16 + n][0] = st[t].m;
            ml[wave][t * 16 + n][1] = st[t].d;
            ml[wave][t * 16 + n][2] = st[t].sum;
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // the references of a column's shares together: its largest m, and what then is the largest m + d less it
        auto tops = [&](int k, float &top, float &scale) {
            top = kLowest, scale = -INFINITY;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) top = fmaxf(top, ml[v][k][0]);
#pragma unroll
            for (int v = 0; v < WAVES; ++v) scale = fmaxf(scale, ml[v][k][0] - top + ml[v][k][1]);
        };
        float top, scale;
        tops(t * 16 + n, top, scale);
        const float mine = __builtin_amdgcn_exp2f(st[t].m - top + st[t].d - scale);
        if (t > 0) __syncthreads();  // the columns before these have been read
        auto share = [&](int of) { return reinterpret_cast<Float4 *>(&red[(of * 16 + n) * kPad + g * 4]); };
        if (WAVES == 8) {  // the upper four first, the others on top
            if (wave >= 4)
#pragma unroll
                for (int d = 0; d < 2 * C; ++d) share(wave - 4)[d * 4] = o[t][d] * mine;
            __syncthreads();
        }
        if (wave < 4)
#pragma unroll
            for (int d = 0; d < 2 * C; ++d) share(wave)[d * 4] = WAVES == 8 ? o[t][d] * mine + share(wave)[d * 4] : o[t][d] * mine;
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * DP / 4; e += WAVES * 64) {
            const int c = e / (DP / 4), d = e % (DP / 4) * 4, k = t * 16 + c;
            Float4 v = *reinterpret_cast<const Float4 *>(&red[c * kPad + d]);
#pragma unroll
            for (int q = 1; q < 4; ++q) v += *reinterpret_cast<const Float4 *>(&red[(q * 16 + c) * kPad + d]);
            float high, total = 0.f, by;
            tops(k, high, by);
#pragma unroll
            for (int q = 0; q < WAVES; ++q) total += ml[q][k][2] * __builtin_amdgcn_exp2f(ml[q][k][0] - high);
            if (parts > 1) {
                keep_part(j, w.slot, NC, k, DP, d, v);
                if (d == 0) keep_sum(j, w.slot, NC, k, high, by, total);
            } else if (tile * NC + k < s.rows * j.group) {
                const int at = tile * NC + k;
                put4(j, s.row0 + at / j.group, head * j.group + at % j.group, d, quotient(v, total, by));
            }
        }
    }
}

// Many rows.  A workgroup has 16 NT columns a wavefront; it goes through the part's units together, two units in LDS
// (keys as bytes, values as FP16, converted once a workgroup), one being read while the next is put there.  Bound by
// issue: of a unit's 32 x 16 weights at 128 dims the matrix instructions take 280 clocks, all else some 250 (a conversion, a
// shift, a fused multiplication, an exponential, half a rounding to FP16 and an addition each), and the wavefronts of a SIMD
// overlap the two in part.  758 rows of 64 heads over 12 000 tokens 251 us, 0.71 PFLOP/s.  Queries in FP16 would save
// the shift and the conversion (13 us less) at twice the rounding errors in the output (4.3e-4 of it, 2.8e-4 now).  A row's second
// reference is 3 us of it.  Prompts from their first token on are further from the floor, since a causal mask leaves
// parts and tiles of different length: 2048 tokens of 32 heads 137 us, 0.25 PFLOP/s, 4096 375 us, 0.37, 16384 3137 us, 0.70.
template <int C, int NT>
__global__ __launch_bounds__(kWaves * 64, NT == 1 && C <= 4 ? 4 : 2) void attend_rows_kernel(Job j) {
    constexpr int NC = 16 * NT * kWaves, DP = C * 32, H = (C + 1) / 2;
    constexpr int kKeys = 2 * H * 1024, kUnitBytes = kKeys + 2 * C * 1024;  // of a unit's keys, with its values
    constexpr int kShare = (C + kWaves - 1) / kWaves;                        // pieces that a wavefront brings, of either
    __shared__ __align__(16) float staged[kWaves * 16 * (DP + 4)];  // queries first, then units: a little less
    static_assert(sizeof(staged) >= 2 * kUnitBytes, "two units");
    const int lane = threadIdx.x & 63, wave = wave_index(), n = lane & 15, g = lane >> 4;
    auto unit_at = [&](int buf) { return reinterpret_cast<uint8_t *>(staged) + buf * kUnitBytes + lane * 16; };
    float *const of_wave = staged + wave * 16 * (DP + 4);
    const Plan plan = make_plan<NC>(j, blockIdx.x == 0 && wave == 0);
    Share w;
    if (!share_of<NC>(j, plan, blockIdx.x, w)) return;
    const Seq &s = w.s;
    const int tile = w.tile, head = w.head, parts = w.parts;
    // units that some column of the workgroup sees
    const Column first = column(j, s, head, tile * NC), last = column(j, s, head, tile * NC + NC - 1);
    const int u0 = max(w.u0, first.lo / kUnit), u1 = min(w.u1, (max(last.hi, 0) + kUnit - 1) / kUnit);
    const int64_t page_bytes = (int64_t)j.c.page * DP;

    // A unit's codes come into registers a unit ahead and go into LDS in the order of the operands, keys as bytes, values as FP16.
    uint4 kc[kShare], vc[kShare];
    PageOf ahead = {}, mine = {};
    auto load = [&](int unit) {
        if ((unit - u0) % 64 == 0) {
            ahead = page_of(j, w.seq, head, unit + lane, u1);
            finish(ahead);
        }
        const int i = (unit - u0) % 64;
        const int64_t off = ((int64_t)max(__builtin_amdgcn_readlane(ahead.id, i), 0) * j.c.kv_heads + head) * page_bytes +
                            (int64_t)__builtin_amdgcn_readlane(ahead.in_page, i) * (kUnit * DP) + lane * 16;
#pragma unroll
        for (int k = 0; k < kShare; ++k) {
            const int c = min(wave + k * kWaves, C - 1);
            kc[k] = *reinterpret_cast<const uint4 *>(j.c.k_codes + off + c * 1024);
            vc[k] = *reinterpret_cast<const uint4 *>(j.c.v_codes + off + c * 1024);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int k = 0; k < kShare; ++k) {
            const int c = wave + k * kWaves;
            if (c >= C) break;
            constexpr uint32_t flip = 0x80808080u;  // code + 128 to the code's own byte
            uint8_t *keys = unit_at(buf) + c / 2 * 2048 + c % 2 * 8, *values = unit_at(buf) + kKeys + c * 2048;
            *reinterpret_cast<uint2 *>(keys) = make_uint2(kc[k].x ^ flip, kc[k].y ^ flip);
            *reinterpret_cast<uint2 *>(keys + 1024) = make_uint2(kc[k].z ^ flip, kc[k].w ^ flip);
            *reinterpret_cast<Half8 *>(values) = halves(vc[k].x, vc[k].y);
            *reinterpret_cast<Half8 *>(values + 1024) = halves(vc[k].z, vc[k].w);
        }
    };
    if (u0 < u1) load(u0);  // on its way while the queries come

    Int4 qh[NT][H], ql[NT][H];
    float factor[NT];
    int lo[NT], hi[NT];
#pragma unroll 1
    for (int tt = 0; tt < NT; ++tt) {  // not unrolled: the code would be long before its first unit
        const int index = tile * NC + (wave * NT + tt) * 16;
        const Column col = column(j, s, head, index + n);
        stage_queries<C>(j, s, head, index, 16, of_wave, lane, 64);
        __syncthreads();
        Int4 high[H], low[H];
        const float f = fixed_query<C>(of_wave, j.scale, col.lo < col.hi, high, low);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (t != tt) continue;
            lo[t] = col.lo, hi[t] = col.hi;
            factor[t] = f;
#pragma unroll
            for (int c = 0; c < H; ++c) qh[t][c] = high[c], ql[t][c] = low[c];
        }
        __syncthreads();
    }
    const int all_hi = __builtin_amdgcn_readlane(hi[0], 0), all_lo = __builtin_amdgcn_readlane(lo[NT - 1], 15);

    Float4 o[NT][2 * C];
    State st[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        st[t] = {kLowest, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < 2 * C; ++d) o[t][d] = Float4{0.f, 0.f, 0.f, 0.f};
    }
    if (C % 2 && wave == 0)  // no dims there: zeros, though the queries are zeros as well
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint2 *>(unit_at(i / 2) + C / 2 * 2048 + 8 + i % 2 * 1024) = make_uint2(0, 0);
    if (u0 < u1) {
        store(0);
        mine = ahead;
        if (u0 + 1 < u1) load(u0 + 1);
    }
    __syncthreads();
    for (int unit = u0; unit < u1; ++unit) {
        const int buf = (unit - u0) & 1, i = (unit - u0) % 64;
        const bool there = __builtin_amdgcn_readlane(mine.id, i) >= 0;
        const float kscale = lane_value(mine.ks, i), log_vs = lane_value(mine.log_vs, i);
        if (unit + 1 < u1) store(buf ^ 1);
        if (unit + 2 < u1) load(unit + 2);
        const uint8_t *from = unit_at(buf);
        __builtin_amdgcn_s_setprio(1);
        float l[NT][8], top[NT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Int4 k[H], sum[NT];
#pragma unroll
            for (int c = 0; c < H; ++c) k[c] = *reinterpret_cast<const Int4 *>(from + c * 2048 + h * 1024);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                sum[t] = Int4{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < H; ++c) sum[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[c], qh[t][c], sum[t], 0, 0, 0);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                sum[t] *= 256;
#pragma unroll
                for (int c = 0; c < H; ++c) sum[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[c], ql[t][c], sum[t], 0, 0, 0);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) l[t][h * 4 + r] = (float)sum[t][r];
        }
        __builtin_amdgcn_s_setprio(0);
        const int t0 = unit * kUnit;
        const bool edge = !there || t0 < all_lo || t0 + kUnit > all_hi;
        bool past = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (edge) {
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int at = t0 + (r >> 2) * 16 + g * 4 + (r & 3);
                    if (!there || at < lo[t] || at >= hi[t]) l[t][r] = -INFINITY;
                }
            }
            top[t] = largest(l[t], logit_factor(factor[t], kscale));
            past |= passes(st[t], top[t], log_vs);
        }
        if (__ballot(past)) move_up<C, NT>(st, top, o, log_vs);
        Half8 p[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) p[t] = weigh(l[t], logit_factor(factor[t], kscale), st[t], log_vs);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const Half8 *of = reinterpret_cast<const Half8 *>(from + kKeys + c * 2048);
            const Half8 v0 = of[0], v1 = of[64];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                o[t][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[t], o[t][2 * c], 0, 0, 0);
                o[t][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[t], o[t][2 * c + 1], 0, 0, 0);
            }
        }
        if (i == 63) mine = ahead;
        __syncthreads();
    }

    // a tile at a time through LDS, so that rows go out whole
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float total = row_sum(st[t].sum);
        const int first_col = (wave * NT + t) * 16;
        if (parts > 1 && g == 0) keep_sum(j, w.slot, NC, first_col + n, st[t].m, st[t].d, total);
#pragma unroll
        for (int d = 0; d < 2 * C; ++d)
            *reinterpret_cast<Float4 *>(of_wave + n * (DP + 4) + d * 16 + g * 4) = parts > 1 ? o[t][d] : quotient(o[t][d], total, st[t].d);
        __syncthreads();
#pragma unroll 1
        for (int e = lane; e < 16 * DP / 4; e += 64) {
            const int c = e / (DP / 4), d = e % (DP / 4) * 4, k = first_col + c, at = tile * NC + k;
            const Float4 v = *reinterpret_cast<const Float4 *>(of_wave + c * (DP + 4) + d);
            if (parts > 1) keep_part(j, w.slot, NC, k, DP, d, v);
            else if (at < s.rows * j.group) put4(j, s.row0 + at / j.group, head * j.group + at % j.group, d, v);
        }
        __syncthreads();
    }
}

// Adds up the parts first, first + step, ... below `parts` of a column, `slot0` being its first part's place and `stride` the way to
// the next: a lane has four dims of every PAR-th of them.  `top` and `scale`: the references of all parts together.
template <int C, int NC>
__device__ __forceinline__ float add_parts(const Job &j, int64_t slot0, int64_t stride, int col, int first, int step, int parts,
                                           float top, float scale, Float4 &acc) {
    constexpr int DP = C * 32, PAR = 64 / (C * 8);
    const int lane = threadIdx.x & 63, mine = lane / (C * 8), d = lane % (C * 8) * 4;
    float total = 0.f;
    acc = Float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = first; p < parts; p += step * PAR) {
        const int at = p + mine * step;
        if (mine >= PAR || at >= parts) continue;
        const int64_t place = (slot0 + at * stride) * NC + col;
        const float *ml = j.part_ml + place * 3;
        const float rise = ml[0] - top, w = __builtin_amdgcn_exp2f(rise + ml[1] - scale);
        const Float4 v = *reinterpret_cast<const Float4 *>(j.part_o + place * DP + d);
        total += __builtin_amdgcn_exp2f(rise) * ml[2];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] += w > 0.f ? w * v[r] : 0.f;  // a part without tokens has no output
    }
    const float mine_total = total;
    const Float4 mine_acc = acc;
#pragma unroll
    for (int k = 1; k < PAR; ++k) {  // the other lanes of these dims, in order behind this one's
        total += __shfl(mine_total, (lane + k * C * 8) & 63);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] += __shfl(mine_acc[r], (lane + k * C * 8) & 63);
    }
    return total;
}

// The references of a column's parts together: their largest m, and what then is the largest m + d less it.
template <int NC>
__device__ __forceinline__ float top_of_parts(const Job &j, int64_t slot0, int64_t stride, int col, int parts, float &scale) {
    const int lane = threadIdx.x & 63;
    auto of = [&](int p) { return j.part_ml + ((slot0 + p * stride) * NC + col) * 3; };
    float m = kLowest, d = 0.f;  // of the first 64 parts, one a lane: read once
    if (lane < parts) m = of(lane)[0], d = of(lane)[1];
    float top = m;
#pragma unroll 1
    for (int p = lane + 64; p < parts; p += 64) top = fmaxf(top, of(p)[0]);
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    scale = m - top + d;
#pragma unroll 1
    for (int p = lane + 64; p < parts; p += 64) scale = fmaxf(scale, of(p)[0] - top + of(p)[1]);
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) scale = fmaxf(scale, __shfl_xor(scale, k));
    return top;
}

// Joins the parts of few rows: SPLIT wavefronts (4 or 1) have a row and query head and share its parts.  `rows_each`: rows that a
// sequence of this kernel has at most.
template <int C, int NC, int SPLIT>
__global__ __launch_bounds__(256) void join_kernel(Job j, int rows_each) {
    __shared__ Float4 outs[4][C * 8];
    __shared__ float sums[4];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int64_t item = SPLIT == 4 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave, seq = item / ((int64_t)rows_each * j.q_heads);
    const int in = (int)(item - seq * rows_each * j.q_heads), r = in / j.q_heads, qh = in % j.q_heads;
    if (seq >= j.n_seq) return;
    bool bad = false;
    const Seq s = sequence(j, seq, bad);
    const int tiles = tiles_of<NC>(j, s);
    if (r >= s.rows || tiles == 0) return;
    const Plan plan = make_plan<NC>(j, false);
    const int parts = parts_of(plan, s);
    if (parts == 1) return;
    const Place place = place_of<NC>(j, plan, [&](const Seq &, int64_t) { return false; }, seq);
    const int index = r * j.group + qh % j.group, col = index % NC;
    const int64_t slot0 = place.kept_before + qh / j.group * tiles + index / NC, stride = (int64_t)tiles * j.c.kv_heads;
    if (slot0 + (parts - 1) * stride >= j.kept) return;
    float scale;
    const float top = top_of_parts<NC>(j, slot0, stride, col, parts, scale);
    Float4 acc;
    const float total = add_parts<C, NC>(j, slot0, stride, col, SPLIT == 4 ? wave : 0, SPLIT, parts, top, scale, acc);
    if (SPLIT == 1) {
        if (lane < C * 8 && lane * 4 < j.c.head_dim) put4(j, s.row0 + r, qh, lane * 4, quotient(acc, total, scale));
        return;
    }
    if (lane < C * 8) outs[wave][lane] = acc;
    if (lane == 0) sums[wave] = total;
    __syncthreads();
    if (wave != 0 || lane >= C * 8 || lane * 4 >= j.c.head_dim) return;
    const float all = sums[0] + sums[1] + sums[2] + sums[3];
    const Float4 o = outs[0][lane] + outs[1][lane] + outs[2][lane] + outs[3][lane];
    put4(j, s.row0 + r, qh, lane * 4, quotient(o, all, scale));
}

// Of many rows: a wavefront has `each` of a row's query heads that share a key / value head.
template <int C, int NC>
__global__ __launch_bounds__(256) void join_rows_kernel(Job j, int each) {
    const int lane = threadIdx.x & 63, runs = (j.group + each - 1) / each;
    const int64_t x = (int64_t)blockIdx.x * 4 + wave_index(), row = x / (j.c.kv_heads * runs);
    const int in = (int)(x - row * (j.c.kv_heads * runs)), head = in / runs, g0 = in % runs * each;
    if (row >= j.n_rows) return;
    const Plan plan = make_plan<NC>(j, false);
    const Place place = place_of<NC>(j, plan, [&](const Seq &s, int64_t) { return s.rows > 0 && row >= s.row0 && row < s.row0 + s.rows; });
    if (place.seq < 0) return;
    bool bad = false;
    const Seq s = sequence(j, place.seq, bad);
    const int parts = parts_of(plan, s), tiles = tiles_of<NC>(j, s);
    if (parts == 1 || tiles == 0) return;
    const int64_t slot = place.kept_before + head * tiles, stride = (int64_t)tiles * j.c.kv_heads;
    if (slot + tiles + (parts - 1) * stride > j.kept) return;
    for (int g = g0; g < min(g0 + each, j.group); ++g) {
        const int index = (int)(row - s.row0) * j.group + g, col = index % NC;
        float scale;
        const float top = top_of_parts<NC>(j, slot + index / NC, stride, col, parts, scale);
        Float4 acc;
        const float total = add_parts<C, NC>(j, slot + index / NC, stride, col, 0, 1, parts, top, scale, acc);
        if (lane < C * 8 && lane * 4 < j.c.head_dim)
            put4(j, row, head * j.group + g, lane * 4, quotient(acc, total, scale));
    }
}

// How a call is launched: the kernel for few rows, for many, or both, each with its columns, workgroups and kept parts.
struct Kernel {
    int nc = 0, target = 0, least = 0;
    bool wide = false;  // 8 wavefronts a workgroup
    int64_t least_cols = 0, most_cols = -1, grid = 0, kept = 0, parts = 1;
};
struct Launches {
    int64_t dp;
    Kernel few, rows;
    size_t o_floats(const Kernel &h) const { return (size_t)(h.kept * h.nc * dp); }
    size_t ml_floats(const Kernel &h) const { return (size_t)(h.kept * h.nc * 3); }
};

// Tiles of 16 columns a wavefront of the kernel for many rows has at most.  Heads of up to 64 and of more than 128 dims are as
// fast or faster with one (us, 1000 rows of 32 heads, 4 to 1: 64 dims, 16384 tokens, 4 tiles 310 and one 299; 192
// dims, 8000 tokens, 2 tiles 331 and one 292).
constexpr int rows_tiles(int64_t c) { return c == 3 || c == 4 ? 3 : 1; }

// A window that no length reaches is none.
int64_t window_of(const cmpq_kv_attention_job *a) { return a->window > INT32_MAX ? 0 : a->window; }

// Units that a sequence's rows see at most.
int64_t most_units(const cmpq_kv_attention_job *a) {
    const int64_t all = cdiv(a->max_length, kUnit), window = window_of(a);
    if (window == 0) return all;
    const int64_t seen = (window + a->max_rows) / kUnit + 2;  // of those of any place in a unit
    return seen < all ? seen : all;
}

int64_t most_tiles(const cmpq_kv_attention_job *a, const Kernel &h) {
    const int64_t group = a->q_heads / a->cache.kv_heads;
    const int64_t most = h.most_cols < a->max_rows * group ? h.most_cols : a->max_rows * group;  // columns of a sequence
    const int64_t by_rows = a->n_rows * group / h.nc + a->n_seq, by_most = a->n_seq * cdiv(most, h.nc);
    return (by_rows < by_most ? by_rows : by_most) * a->cache.kv_heads;
}

void size_up(const cmpq_kv_attention_job *a, Kernel &h) {
    const int64_t tiles = most_tiles(a, h), parts = cdiv(most_units(a), h.least);
    h.grid = tiles;
    if (parts > 1) {
        const int64_t full = tiles * parts;
        h.grid = full < tiles + 2 * h.target ? full : tiles + 2 * h.target;
        h.kept = full < 2 * h.target ? full : 2 * h.target;
        h.parts = parts;
    }
}

// Where the kernel for many rows takes those tiles: from so many units of theirs on.  Below, one a wavefront and four
// wavefronts a SIMD in place of two.  us, three tiles and one, heads of 128 dims: 1000 rows over 16384 tokens, 4 to 1 (86 000
// units), 320 and 385; 1024 over 4096, 8 to 1 (44 000), 239 and 200; 2048 over 2048 of 32 heads (22 500) 164 and 133.
constexpr int64_t kManyUnits = 50000;

// Where sequences of single rows among ones of many have the kernel for few rows: from so many units of theirs on.  Below, its
// two launches cost more than it saves.  us, with it and without: a sequence of 3000 tokens beside 700 rows (750 units)
// 133 and 119, 8 of up to 4096 beside 8 chunks (15 000) 118 and 107, 16 beside 16 (32 000) 134 and 165, 16 of up to 8192
// beside 16 of 64 rows (63 000) 156 and 225.
constexpr int64_t kApartUnits = 20000;

Launches plan_launches(const cmpq_kv_attention_job *a) {
    Launches l;
    const int64_t c = cdiv(a->cache.head_dim, 32), group = a->q_heads / a->cache.kv_heads, cols = a->max_rows * group;
    l.dp = c * 32;
    // Columns that the kernel for few rows takes at most, as registers allow.  us, it and the one for many rows: 48 columns of 128
    // dims, 8 heads, 8000 tokens 26.6 and 30.4, 32 such sequences 123 and 153 (64 of 1000 tokens 46.6 and 41.1); 32 columns of
    // 192 dims 26.9 and 39.4.
    const int64_t few = c <= 4 ? 48 : 32;
    if (cols <= few) {
        l.few.nc = (int)cdiv(cols, 16) * 16;
        l.few.least_cols = 1;
        l.few.most_cols = few;
    } else if (group <= few && (a->n_seq - 1) * a->cache.kv_heads * most_units(a) >= kApartUnits) {
        l.few.nc = (int)cdiv(group, 16) * 16;
        l.few.least_cols = 1;
        l.few.most_cols = l.few.nc;
    }
    if (cols > few) {
        l.rows.nc = 16 * kWaves * rows_tiles(c);
        l.rows.least_cols = l.few.most_cols > 0 ? l.few.most_cols + 1 : 1;
        l.rows.most_cols = INT64_MAX;
        if (most_tiles(a, l.rows) * most_units(a) < kManyUnits) l.rows.nc = 16 * kWaves;
    }
    l.few.target = 1024, l.few.least = 8;
    // Short sequences in one part, by 8 wavefronts where that leaves compute units free: a part more costs the launch that
    // joins them.  us, one part and several: 32 heads, 1000 tokens 11.8 and 13.5, 1300 13.0 and 13.9, 2000 15.8 and 14.1; 32
    // sequences of up to 1300 15.0 and 20.7.  8 wavefronts and 4: 2000 tokens 15.8 and 17.8, 64 sequences (512 tiles) 28.5 and 26.4.
    if (l.few.nc && most_units(a) <= 48) {
        l.few.least = 48;
        l.few.wide = most_tiles(a, l.few) < 512;
    }
    l.rows.target = l.rows.nc == 16 * kWaves && c <= 4 ? 1024 : 512;  // workgroups that run at once
    l.rows.least = 16;
    if (l.few.nc) size_up(a, l.few);
    if (l.rows.nc) size_up(a, l.rows);
    return l;
}

// Sizes alone.  Columns of a tile, items of a join and workgroups are counted in 32 bits.
int check_sizes(const cmpq_kv_attention_job *a) {
    if (a->n_seq < 0 || a->n_rows < 0 || a->max_rows < 0 || a->max_length < 0 || a->ld_table < 0 || a->window < 0)
        return CMPQ_EINVAL;
    if (a->cache.kv_heads < 1 || a->q_heads < 1 || a->q_heads % a->cache.kv_heads) return CMPQ_EINVAL;
    if (!cmpq_kv_page_bytes(a->cache.head_dim, a->cache.page)) return CMPQ_ESHAPE;
    if (a->n_seq > INT32_MAX || a->n_rows > INT32_MAX || a->max_length > INT32_MAX - kUnit || a->q_heads > 65535 ||
        a->ld_table > INT32_MAX || a->max_rows > INT32_MAX || a->n_rows * a->q_heads > ((int64_t)1 << 32))
        return CMPQ_ESHAPE;
    const int64_t rows = a->max_rows < a->n_rows ? a->max_rows : a->n_rows;
    if (rows * (a->q_heads / a->cache.kv_heads) > INT32_MAX - 1024 || a->n_seq * 48 * a->q_heads > INT32_MAX) return CMPQ_ESHAPE;
    return CMPQ_OK;
}

int check_job(const cmpq_kv_attention_job *a) {
    if (!a) return CMPQ_EINVAL;
    if (int rc = check_cache(a->cache)) return rc;
    if (!serving_dtype(a->q_dtype) || (a->o_dtype != CMPQ_F16 && a->o_dtype != CMPQ_BF16)) return CMPQ_EINVAL;
    if (int rc = check_sizes(a)) return rc;
    return check_rotation(&a->rotation, a->cache.head_dim);
}

template <int C, int NT>
void launch_few(const Job &j, const Kernel &h, hipStream_t st) {
    if constexpr (C * NT <= 8) {
        if (h.wide) attend_kernel<C, NT, 8><<<dim3((unsigned)h.grid), 512, 0, st>>>(j);
        else attend_kernel<C, NT, 4><<<dim3((unsigned)h.grid), 256, 0, st>>>(j);
    } else {
        attend_kernel<C, NT, 4><<<dim3((unsigned)h.grid), 256, 0, st>>>(j);
    }
    if (!h.kept) return;
    const int64_t each = h.most_cols / j.group < j.max_rows ? h.most_cols / j.group : j.max_rows;
    const int64_t items = j.n_seq * each * j.q_heads;
    // us, 4 wavefronts and 1: 2 sequences of 64 heads (up to 80 parts) 9.0 and 12.4, 64 of them (3 parts) 12.5 and 6.6
    if (items < 2048) join_kernel<C, NT * 16, 4><<<dim3((unsigned)items), 256, 0, st>>>(j, (int)each);
    else join_kernel<C, NT * 16, 1><<<dim3((unsigned)cdiv(items, 4)), 256, 0, st>>>(j, (int)each);
}

template <int C, int NT>
void launch_rows(const Job &j, const Kernel &h, hipStream_t st) {
    attend_rows_kernel<C, NT><<<dim3((unsigned)h.grid), kWaves * 64, 0, st>>>(j);
    if (!h.kept) return;
    // heads one after the other only where there are wavefronts enough all the same
    const int64_t all = cdiv(j.n_rows * j.q_heads, 4096), each = all < j.group ? all : j.group;
    const int64_t waves = j.n_rows * j.c.kv_heads * cdiv(j.group, each);
    join_rows_kernel<C, NT * 16 * kWaves><<<dim3((unsigned)cdiv(waves, 4)), 256, 0, st>>>(j, (int)each);
}

template <int C>
void launch(Job j, const Launches &l, WsCarver &w, hipStream_t st) {
    auto take = [&](const Kernel &h) {
        j.target = h.target, j.least = h.least, j.least_cols = h.least_cols, j.most_cols = h.most_cols, j.kept = h.kept;
        j.most_parts = (int)h.parts;
        j.part_o = w.take<float>(l.o_floats(h));
        j.part_ml = w.take<float>(l.ml_floats(h));
    };
    if (l.rows.nc) {
        take(l.rows);
        if (l.rows.nc == 16 * kWaves) launch_rows<C, 1>(j, l.rows, st);
        else if constexpr (rows_tiles(C) > 1) launch_rows<C, rows_tiles(C)>(j, l.rows, st);
    }
    if (l.few.nc) {
        take(l.few);
        if (l.few.nc == 16) launch_few<C, 1>(j, l.few, st);
        else if (l.few.nc == 32) launch_few<C, 2>(j, l.few, st);
        else if constexpr (C <= 4) launch_few<C, 3>(j, l.few, st);
    }
}

size_t workspace_of(const Launches &l) {
    WsCarver w(nullptr);
    for (const Kernel *h : {&l.rows, &l.few}) {
        if (!h->nc) continue;
        w.take<float>(l.o_floats(*h));
        w.take<float>(l.ml_floats(*h));
    }
    return w.need() > 256 ? w.need() : 256;
}

}  // namespace

extern "C" size_t cmpq_kv_attention_workspace(const cmpq_kv_attention_job *a) {
    return a && check_sizes(a) == CMPQ_OK ? workspace_of(plan_launches(a)) : 0;
}

extern "C" int cmpq_kv_attention(const cmpq_kv_attention_job *a, void *ws, size_t ws_bytes, void *stream) {
    if (int rc = check_job(a)) return rc;
    if (a->n_seq == 0 || a->n_rows == 0 || a->max_rows == 0)
        return cmpq_flag_named_rows(a->cu_rows, a->n_seq, a->status, static_cast<hipStream_t>(stream));
    if (!a->page_table || !a->lengths || !a->cu_rows || !a->Q.ptr || !a->O.ptr) return CMPQ_EINVAL;
    const Launches l = plan_launches(a);
    if (l.few.grid > INT32_MAX || l.rows.grid > INT32_MAX) return CMPQ_ESHAPE;
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < workspace_of(l)) return CMPQ_EWORKSPACE;
    WsCarver w(ws);
    Job j = {};
    j.c = a->cache;
    j.table = a->page_table, j.lengths = a->lengths, j.cu = a->cu_rows;
    j.ld_table = a->ld_table, j.n_seq = a->n_seq, j.n_rows = a->n_rows, j.max_rows = a->max_rows;
    j.max_length = a->cache.n_pages > 0 ? a->max_length : 0;
    j.Q = a->Q, j.O = a->O, j.q_dtype = a->q_dtype, j.o_dtype = a->o_dtype, j.q_heads = a->q_heads;
    j.group = a->q_heads / a->cache.kv_heads;
    j.scale = a->softmax_scale, j.causal = a->causal, j.window = window_of(a), j.rot = a->rotation, j.status = a->status;
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (l.dp / 32) {
        case 1: launch<1>(j, l, w, st); break;
        case 2: launch<2>(j, l, w, st); break;
        case 3: launch<3>(j, l, w, st); break;
        case 4: launch<4>(j, l, w, st); break;
        case 5: launch<5>(j, l, w, st); break;
        case 6: launch<6>(j, l, w, st); break;
        case 7: launch<7>(j, l, w, st); break;
        default: launch<8>(j, l, w, st); break;
    }
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
