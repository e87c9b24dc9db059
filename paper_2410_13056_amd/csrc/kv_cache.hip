// The paged cache in 8 bits: new tokens in (keys turned by position on the way) and values back.
// A workgroup takes one page of one sequence for one head, keys or values: a scale belongs to a page and head, so
// whoever finds the page's new largest magnitude also writes its codes, and nobody else touches them.  The new values are
// in registers between the two: they are read once from memory.
//
// Bound.  Prompts: 5701 tokens of 32 heads, 128 dims, FP16, 140 MB in 47 us (3.0 TB/s): vector instructions
// keep the units busy for 68 % of it (25 a value: turn, magnitude, code, addresses, and the search for the
// page), stores in whole lines took 5 us off.  Read back: 30 us, 4.7 TB/s, what a large copy reaches.  Steps: 64 sequences of
// one token, 8 heads, 6.4 us and 9 us back: a chain of loads (lengths, page table, scale, codes).  That is a step in which no
// page's scale grows.  With fresh tokens some do in nearly every step, and the launch waits for the codes that they hold to be
// rounded again, word by word (hold_item): the mean of 64 steps in one graph 13.5 us, of the same step 64 times 5.8.
#include "serving.h"

namespace {

struct Page {
    int64_t seq;     // sequence, -1: there is no such page
    int64_t begin;   // its first token's position
    int64_t first;   // position of the sequence's first row
    int64_t row0;    // that row
    int from, to;    // rows of this call: the page's tokens from .. to-1
};

// Rows of sequence i, within the call's.
__device__ __forceinline__ int64_t rows_of(const cmpq_kv_rows &r, int64_t i, int64_t &row0, bool &bad) {
    const int64_t a = r.cu_rows[i], b = r.cu_rows[i + 1];
    row0 = min(max(a, (int64_t)0), r.n_rows);
    const int64_t end = min(max(b, row0), r.n_rows);
    bad |= a != row0 || b != end;
    return end - row0;
}

// The `x`-th of the pages that the call's rows lie in, sequence after sequence; `x` is the same in all lanes of the
// wavefront, 64 sequences are counted at a time.  With `status` the wavefront looks all sequences over.
__device__ __forceinline__ Page find_page(const cmpq_kv_rows &r, int page, int64_t x, int32_t *status) {
    const int lane = threadIdx.x & 63;
    Page p = {-1, 0, 0, 0, 0, 0};
    int64_t before = 0;
    for (int64_t base = 0; base < r.n_seq; base += 64) {
        const int64_t i = base + lane;
        int64_t row0 = 0, n = 0, first = 0;
        bool bad = false;
        if (i < r.n_seq) {
            n = rows_of(r, i, row0, bad);
            first = r.first[i];
            bad |= first < 0;
            if (first < 0) n = 0;
            const int64_t room = r.ld_table * page - first;  // tokens that the table has pages for
            if (n > 0 && n > room) {
                bad = true;
                n = max(room, (int64_t)0);
            }
        }
        if (bad && status) atomicOr(status, CMPQ_STATUS_RANGE);
        const uint32_t pages = n > 0 ? (uint32_t)((first + n - 1) / page - first / page + 1) : 0;
        const uint32_t incl = wave_scan_incl_u32(pages);
        const uint64_t past = __ballot(before + incl > x);
        if (past && p.seq < 0) {
            const int l = __builtin_ctzll(past);
            const int64_t seq_first = __shfl(first, l), seq_rows = __shfl(n, l);
            const int64_t nth = x - before - (int64_t)(__shfl(incl, l) - __shfl(pages, l));
            p.seq = base + l;
            p.first = seq_first;
            p.row0 = __shfl(row0, l);
            p.begin = (seq_first / page + nth) * page;
            p.from = (int)(max(seq_first, p.begin) - p.begin);
            p.to = (int)(min(seq_first + seq_rows, p.begin + page) - p.begin);
            if (!status) return p;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
    return p;
}

// One wavefront of the launch.
__device__ __forceinline__ bool looks_over() {
    return (blockIdx.x | blockIdx.y | blockIdx.z) == 0 && wave_index() == 0;
}

// An item is four tokens next to each other by eight dims, a lane's share: in the stored order its keys are four runs of 8
// bytes, its values eight of 4 bytes, which no other item has a part in.
struct Item {
    int tok, d;      // first of each
    uint8_t *at;     // keys: of the first token (the others 16 bytes apart); values: of the first dim (16 bytes apart)
};

// Items e -> (four tokens, octet of dims), without a division: e * octets stays below 2^18 (1024 tokens of 256 dims), so the
// product by 2^20 / octets, rounded up, has the right whole part.
struct Octets {
    uint32_t n, inverse;
    __device__ __forceinline__ explicit Octets(int head_dim) : n((head_dim + 31) / 32 * 4), inverse((1u << 20) / n + 1) {}
};

template <bool KEYS>
__device__ __forceinline__ Item item_of(uint32_t e, const Octets &octets, uint8_t *codes) {
    const uint32_t four = e * octets.inverse >> 20, tok = four * 4, dim = (e - four * octets.n) * 8, t = tok % 32, d = dim % 32;
    Item it;
    it.tok = (int)tok;
    it.d = (int)dim;
    it.at = codes + (tok / 32 * (octets.n / 4) + dim / 32) * 1024 +
            (KEYS ? d / 8 * 256 + t % 16 * 16 + t / 16 * 8 : t % 16 / 4 * 256 + d % 16 * 16 + d / 16 * 8 + t / 16 * 4);
    return it;
}

// The new values of an item: 0 for tokens that are not new and for dims beyond the head.  WHOLE: eight dims are all there or
// none, and turn by eight.
template <typename T, bool KEYS, bool WHOLE>
__device__ __forceinline__ void load_item(const cmpq_kv_cache &c, const Page &pg, const cmpq_heads &in, const cmpq_rotation &rot,
                                          int head, const Item &it, float (&x)[4][8]) {
    const int64_t t0 = pg.begin + it.tok, turn = min(t0, rot.positions - 1), half = rot.dims >> 1;
    const int more = (int)min((int64_t)3, rot.positions - 1 - turn);  // rows of the tables after this one
    const T *p0 = static_cast<const T *>(in.ptr) + head * in.head_stride + (pg.row0 + t0 - pg.first) * in.row_stride;
    const int64_t row = turn * half;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int tok = it.tok + r;
        const T *p = p0 + r * in.row_stride;
        const bool is_new = tok >= pg.from && tok < pg.to;
        if (WHOLE && is_new && it.d < c.head_dim) {
            if (KEYS) load_turned(p, it.d, rot, row + min(r, more) * (int)half, x[r]);
            else load_f32<T, 8>(p + it.d, x[r]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[r][i] = 0.f;
                if (!WHOLE && is_new && it.d + i < c.head_dim) x[r][i] = KEYS ? turned(p, it.d + i, rot, turn + min(r, more)) : (float)p[it.d + i];
            }
        }
    }
}

// Codes of an item, none of them NaN: for keys two words a token, for values one a dim.
template <bool KEYS>
__device__ __forceinline__ void code_item(const float (&x)[4][8], float inv, uint32_t (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) b[k] = code_byte<128>(KEYS ? x[i / 2][i % 2 * 4 + k] : x[k][i], inv);
        w[i] = low_bytes(b[0], b[1], b[2], b[3]);
    }
}

// Where byte `at` of staged codes lies in LDS: 16 bytes stay together, other lanes' of one instruction go to other banks.
__device__ __forceinline__ int staged_at(int at) { return at ^ (at >> 4 & 0xf0); }

template <bool KEYS>
__device__ __forceinline__ void stage_item(uint8_t *staged, int at, const uint32_t (&w)[8]) {
    if (KEYS) {
#pragma unroll
        for (int r = 0; r < 4; ++r) *reinterpret_cast<uint2 *>(staged + staged_at(at + r * 16)) = make_uint2(w[2 * r], w[2 * r + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<uint32_t *>(staged + staged_at(at + i * 16)) = w[i];
    }
}

// Codes of an item's new tokens into the page; the bytes of others stay.
template <bool KEYS>
__device__ __forceinline__ void store_item(const Page &pg, const Item &it, const uint32_t (&w)[8]) {
    if (KEYS) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (it.tok + r >= pg.from && it.tok + r < pg.to) *reinterpret_cast<uint2 *>(it.at + r * 16) = make_uint2(w[2 * r], w[2 * r + 1]);
    } else {
        uint32_t keep = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (it.tok + r < pg.from || it.tok + r >= pg.to) keep |= 255u << (8 * r);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t *at = reinterpret_cast<uint32_t *>(it.at + i * 16);
            *at = keep ? (*at & keep) | (w[i] & ~keep) : w[i];
        }
    }
}

// Codes of an item's tokens before the new ones, times `again`.
template <bool KEYS>
__device__ __forceinline__ void hold_item(const Page &pg, const Item &it, float again) {
    const int n = min(4, pg.from - it.tok);  // tokens
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        uint32_t *at = reinterpret_cast<uint32_t *>(it.at + (KEYS ? i / 2 * 16 + i % 2 * 4 : i * 16));
        if (KEYS && i / 2 >= n) break;
        const uint32_t had = *at;
        uint32_t w = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int code = (int)((had >> (8 * b)) & 255) - 128;
            w |= (uint32_t)((KEYS || b < n ? (int)rintf((float)code * again) : code) + 128) << (8 * b);
        }
        *at = w;
    }
}

// Blocks of 32 tokens that a workgroup takes at once, one item a lane.
template <int THREADS>
__device__ __forceinline__ int blocks_at_once(int chunks) {
    return max(1, THREADS / (32 * chunks));
}

// The new values are read once where each lane has at most one item, else again for their codes.  Codes of whole blocks of 32
// tokens go out through LDS, 1 KB in order a wavefront; written from the lanes that make them, 4 or 8 bytes each, they
// would take up a line of the cache behind each time.
template <typename T, bool KEYS, bool WHOLE, int THREADS>
__device__ __forceinline__ void append_page(const cmpq_kv_cache &c, const Page &pg, int64_t id, int head, const cmpq_heads &in,
                                            const cmpq_rotation &rot, int32_t *status, float *scratch, uint8_t *staged) {
    constexpr bool kStaged = THREADS == 256;
    const Octets octets(c.head_dim);
    const int chunks = (int)octets.n / 4, block_items = chunks * 32, block_bytes = chunks * 1024;
    uint8_t *codes = (KEYS ? c.k_codes : c.v_codes) + (id * c.kv_heads + head) * (int64_t)(c.page * chunks * 32);
    float *scale = (KEYS ? c.k_scale : c.v_scale) + id * c.kv_heads + head;
    if (threadIdx.x == 0) scratch[THREADS / 64] = pg.from > 0 ? *scale : 0.f;
    const int step = kStaged ? blocks_at_once<THREADS>(chunks) * block_items : THREADS;
    const int start = kStaged ? pg.from / 32 * block_items : pg.from / 4 * (int)octets.n, e0 = pg.from / 4 * (int)octets.n;
    const int e1 = (pg.to + 3) / 4 * (int)octets.n;
    const bool once = e1 - start <= step;
    const int staged_bytes = step / 32 * 1024;
    const int whole0 = (pg.from + 31) / 32, whole1 = pg.to / 32;  // whole blocks
    float x[4][8];
    Largest largest;
    bool bad = false;
    auto has = [&](int e) { return (int)threadIdx.x < step && e >= e0 && e < e1; };
    auto look = [&](int e) {
        load_item<T, KEYS, WHOLE>(c, pg, in, rot, head, item_of<KEYS>(e, octets, codes), x);
        Largest here;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) here.add(x[r][i]);
        if (here.bad()) {
            bad = true;
            here.bits = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) here.add_finite(x[r][i]);
        }
        largest.bits = max(largest.bits, here.bits);
    };
    if (once) {
        if (has(start + threadIdx.x)) look(start + threadIdx.x);
    } else {
#pragma unroll 1
        for (int base = start; base < e1; base += step)
            if (has(base + threadIdx.x)) look(base + threadIdx.x);
    }
    if (bad && status) atomicOr(status, CMPQ_STATUS_NONFINITE);
    if (KEYS && rot.cos && threadIdx.x == 0 && status && pg.begin + pg.to > rot.positions) atomicOr(status, CMPQ_STATUS_RANGE);
    const float most = block_max(largest.most(), scratch), old = scratch[THREADS / 64], now = fmaxf(old, code_scale(most));
    const float inv = 1.f / now;
    if (threadIdx.x == 0) *scale = now;
    if (pg.from > 0 && now != old) {
        for (int e = threadIdx.x; e < (pg.from + 3) / 4 * (int)octets.n; e += THREADS)
            hold_item<KEYS>(pg, item_of<KEYS>(e, octets, codes), old * inv);
        __syncthreads();  // an item of both is held first, by whichever lane
    }
    auto put = [&](int e, int byte) {
        const Item it = item_of<KEYS>(e, octets, codes);
        if (bad)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[r][i] = no_nan(x[r][i]);
        uint32_t w[8];
        code_item<KEYS>(x, inv, w);
        if (kStaged && it.tok / 32 >= whole0 && it.tok / 32 < whole1) stage_item<KEYS>(staged, (int)(it.at - codes) - byte, w);
        else store_item<KEYS>(pg, it, w);
    };
    auto copy_out = [&](int byte) {
        __syncthreads();
        const int end = min(staged_bytes, whole1 * block_bytes - byte);
        for (int at = max(0, whole0 * block_bytes - byte) + threadIdx.x * 16; at < end; at += THREADS * 16)
            *reinterpret_cast<uint4 *>(codes + byte + at) = *reinterpret_cast<const uint4 *>(staged + staged_at(at));
    };
    if (once) {
        if (has(start + threadIdx.x)) put(start + threadIdx.x, start / 32 * 1024);
        if (kStaged) copy_out(start / 32 * 1024);
    } else {
#pragma unroll 1
        for (int base = start, byte = start / 32 * 1024; base < e1; base += step, byte += staged_bytes) {  // codes begin there
            if (has(base + threadIdx.x)) {
                load_item<T, KEYS, WHOLE>(c, pg, in, rot, head, item_of<KEYS>(base + threadIdx.x, octets, codes), x);
                put(base + threadIdx.x, byte);
            }
            if (!kStaged) continue;
            copy_out(byte);
            __syncthreads();
        }
    }
}

// THREADS: 256, or a wavefront where sequences have up to 4 rows on average (64 sequences of one token 7.4 us, with 256 8.6).
template <typename T, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void append_kernel(cmpq_kv_cache c, cmpq_kv_rows r, cmpq_heads K, cmpq_heads V,
                                                          cmpq_rotation rot, int32_t *status) {
    __shared__ float scratch[THREADS / 64 + 1];
    __shared__ __align__(16) uint8_t staged[THREADS == 256 ? 8192 : 16];
    const Page pg = find_page(r, c.page, blockIdx.x, looks_over() ? status : nullptr);
    if (pg.seq < 0) return;
    const int64_t id = r.page_table[pg.seq * r.ld_table + pg.begin / c.page];
    if (id < 0 || id >= c.n_pages) {
        if (threadIdx.x == 0 && status) atomicOr(status, CMPQ_STATUS_RANGE);
        return;
    }
    if (blockIdx.z == 0) append_page<T, true, WHOLE, THREADS>(c, pg, id, blockIdx.y, K, rot, status, scratch, staged);
    else append_page<T, false, WHOLE, THREADS>(c, pg, id, blockIdx.y, V, rot, status, scratch, staged);
}

template <typename T, bool KEYS, int THREADS>
__device__ void read_page(const cmpq_kv_cache &c, const Page &pg, int64_t id, int head, const cmpq_heads &out) {
    const Octets octets(c.head_dim);
    const int dim = c.head_dim, chunks = (int)octets.n / 4;
    uint8_t *codes = (KEYS ? c.k_codes : c.v_codes) + (id * c.kv_heads + head) * (int64_t)(c.page * chunks * 32);
    const float scale = (KEYS ? c.k_scale : c.v_scale)[id * c.kv_heads + head];
    T *base = static_cast<T *>(out.ptr) + head * out.head_stride;
    const int e0 = pg.from / 4 * (int)octets.n, e1 = (pg.to + 3) / 4 * (int)octets.n;
    for (int e = e0 + threadIdx.x; e < e1; e += THREADS) {
        const Item it = item_of<KEYS>(e, octets, codes);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = *reinterpret_cast<const uint32_t *>(it.at + (KEYS ? i / 2 * 16 + i % 2 * 4 : i * 16));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int tok = it.tok + r;
            if (tok < pg.from || tok >= pg.to) continue;
            T *p = base + (pg.row0 + pg.begin + tok - pg.first) * out.row_stride + it.d;
            typedef T T8 __attribute__((ext_vector_type(8)));
            typedef T8 Any __attribute__((aligned(sizeof(T))));
            T8 v;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t code = KEYS ? w[2 * r + i / 4] >> (8 * (i & 3)) : w[i] >> (8 * r);
                v[i] = (T)((float)((int)(code & 255) - 128) * scale);
            }
            if (it.d + 8 <= dim) {
                *reinterpret_cast<Any *>(p) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (it.d + i < dim) p[i] = v[i];
            }
        }
    }
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void read_kernel(cmpq_kv_cache c, cmpq_kv_rows r, cmpq_heads K, cmpq_heads V,
                                                        int32_t *status) {
    const Page pg = find_page(r, c.page, blockIdx.x, looks_over() ? status : nullptr);
    if (pg.seq < 0) return;
    const int64_t id = r.page_table[pg.seq * r.ld_table + pg.begin / c.page];
    if (id < 0 || id >= c.n_pages) {
        if (threadIdx.x == 0 && status) atomicOr(status, CMPQ_STATUS_RANGE);
        return;
    }
    if (blockIdx.z == 0) read_page<T, true, THREADS>(c, pg, id, blockIdx.y, K);
    else read_page<T, false, THREADS>(c, pg, id, blockIdx.y, V);
}

int check_rows(const cmpq_kv_cache *c, const cmpq_kv_rows *r, const cmpq_heads *K, const cmpq_heads *V, int dtype) {
    if (!c || !r || !K || !V || !serving_dtype(dtype)) return CMPQ_EINVAL;
    if (int rc = check_cache(*c)) return rc;
    if (r->n_seq < 0 || r->n_rows < 0 || r->ld_table < 0) return CMPQ_EINVAL;
    if (r->n_seq > INT32_MAX || r->n_rows > INT32_MAX || r->ld_table > INT32_MAX) return CMPQ_ESHAPE;
    if (r->n_seq == 0 || r->n_rows == 0 || r->ld_table == 0) return CMPQ_OK;
    if (!r->page_table || !r->first || !r->cu_rows || !K->ptr || !V->ptr) return CMPQ_EINVAL;
    return CMPQ_OK;
}

// Workgroups: a sequence with n > 0 rows lies in at most n, and at most n / page + 2 pages.
dim3 page_grid(const cmpq_kv_cache &c, const cmpq_kv_rows &r) {
    const int64_t most = r.n_rows / c.page + 2 * r.n_seq;
    return dim3((unsigned)(most < r.n_rows ? most : r.n_rows), (unsigned)c.kv_heads, 2);
}

__global__ __launch_bounds__(64) void named_rows_kernel(const int32_t *cu, int64_t n_seq, int32_t *status) {
    for (int64_t i = threadIdx.x; i < n_seq; i += 64)
        if (cu[i + 1] > cu[i]) atomicOr(status, CMPQ_STATUS_RANGE);
}

}  // namespace

int cmpq_flag_named_rows(const int32_t *cu, int64_t n_seq, int32_t *status, hipStream_t stream) {
    if (!status || !cu || n_seq < 1) return CMPQ_OK;
    named_rows_kernel<<<1, 64, 0, stream>>>(cu, n_seq, status);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

extern "C" size_t cmpq_kv_page_bytes(int head_dim, int page) {
    if (head_dim < 1 || head_dim > 256 || page < 32 || page > 1024 || page % 32) return 0;
    return (size_t)page * 32 * ((head_dim + 31) / 32);
}

extern "C" int cmpq_kv_append(const cmpq_kv_cache *cache, const cmpq_kv_rows *rows, const cmpq_heads *K,
                              const cmpq_heads *V, int dtype, const cmpq_rotation *rotation, int32_t *status,
                              void *stream) {
    if (int rc = check_rows(cache, rows, K, V, dtype)) return rc;
    if (int rc = check_rotation(rotation, cache->head_dim)) return rc;
    if (rows->n_seq == 0 || rows->n_rows == 0 || rows->ld_table == 0)
        return cmpq_flag_named_rows(rows->cu_rows, rows->n_seq, status, static_cast<hipStream_t>(stream));
    const cmpq_rotation rot = rotation ? *rotation : cmpq_rotation{};
    const dim3 grid = page_grid(*cache, *rows);
    const bool whole = cache->head_dim % 8 == 0 && turns_by_eight(rot), wavefronts = whole && rows->n_rows <= 4 * rows->n_seq;
    if (!one_launch(grid.x, wavefronts ? 64 : 256)) return CMPQ_ESHAPE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](auto like) {
        using T = decltype(like);
        if (!whole) append_kernel<T, false, 256><<<grid, 256, 0, st>>>(*cache, *rows, *K, *V, rot, status);
        else if (!wavefronts) append_kernel<T, true, 256><<<grid, 256, 0, st>>>(*cache, *rows, *K, *V, rot, status);
        else append_kernel<T, true, 64><<<grid, 64, 0, st>>>(*cache, *rows, *K, *V, rot, status);
    };
    if (dtype == CMPQ_F16) launch(_Float16());
    else if (dtype == CMPQ_BF16) launch(__bf16());
    else launch(float());
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

extern "C" int cmpq_kv_read(const cmpq_kv_cache *cache, const cmpq_kv_rows *rows, const cmpq_heads *K,
                            const cmpq_heads *V, int dtype, int32_t *status, void *stream) {
    if (int rc = check_rows(cache, rows, K, V, dtype)) return rc;
    if (rows->n_seq == 0 || rows->n_rows == 0 || rows->ld_table == 0)
        return cmpq_flag_named_rows(rows->cu_rows, rows->n_seq, status, static_cast<hipStream_t>(stream));
    const dim3 grid = page_grid(*cache, *rows);
    if (!one_launch(grid.x, 256)) return CMPQ_ESHAPE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == CMPQ_F16) read_kernel<_Float16, 256><<<grid, 256, 0, st>>>(*cache, *rows, *K, *V, status);
    else if (dtype == CMPQ_BF16) read_kernel<__bf16, 256><<<grid, 256, 0, st>>>(*cache, *rows, *K, *V, status);
    else read_kernel<float, 256><<<grid, 256, 0, st>>>(*cache, *rows, *K, *V, status);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
