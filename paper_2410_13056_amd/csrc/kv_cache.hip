// The paged cache in 8 bits: new tokens in (keys turned by position on the way) and values back.
// A workgroup takes one page of one sequence for one head, keys or values: a scale belongs to a page and head, so
// whoever finds the page's new largest magnitude also writes its codes, and nobody else touches them.
#include "serving.h"

namespace {

constexpr int kThreads = 256;

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
            if (n > room) {
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

// Token and dim of byte j of the 8-byte half `h` of the 16 bytes that lane l has of a piece.
template <bool KEYS>
__device__ __forceinline__ int token_in_piece(int l, int h, int j) {
    return KEYS ? 16 * h + (l & 15) : 16 * (j >> 2) + 4 * (l >> 4) + (j & 3);
}
template <bool KEYS>
__device__ __forceinline__ int dim_in_piece(int l, int h, int j) {
    return KEYS ? 8 * (l >> 4) + j : 16 * h + (l & 15);
}

template <typename T, bool KEYS>
__device__ void append_page(const cmpq_kv_cache &c, const Page &pg, int64_t id, int head, const cmpq_heads &in,
                            const cmpq_rotation &rot, int32_t *status, float *scratch) {
    const int dim = c.head_dim, chunks = (dim + 31) / 32;
    const T *base = static_cast<const T *>(in.ptr) + head * in.head_stride;
    auto value = [&](int tok, int d) {
        const int64_t at = pg.begin + tok;
        const T *p = base + (pg.row0 + at - pg.first) * in.row_stride;
        return KEYS ? turned(p, d, rot, min(at, rot.positions - 1)) : (float)p[d];
    };
    float most = 0.f;
    bool bad = false;
    const int n = pg.to - pg.from;
    for (int e = threadIdx.x; e < n * dim; e += kThreads) most = fmaxf(most, finite_abs(value(pg.from + e / dim, e % dim), bad));
    if (bad && status) atomicOr(status, CMPQ_STATUS_NONFINITE);
    if (KEYS && rot.cos && threadIdx.x == 0 && status && pg.begin + pg.to > rot.positions)
        atomicOr(status, CMPQ_STATUS_RANGE);
    most = block_max(most, scratch);
    float *scale = (KEYS ? c.k_scale : c.v_scale) + id * c.kv_heads + head;
    const float old = pg.from > 0 ? *scale : 0.f;
    const float now = fmaxf(old, code_scale(most)), inv = 1.f / now, again = old * inv;
    __syncthreads();  // everybody has the old scale
    if (threadIdx.x == 0) *scale = now;
    uint8_t *codes = (KEYS ? c.k_codes : c.v_codes) + (id * c.kv_heads + head) * (int64_t)(c.page * chunks * 32);
    const bool grown = pg.from > 0 && now != old;
    const int pieces = c.page / 32 * chunks;
    for (int e = threadIdx.x; e < pieces * 128; e += kThreads) {  // 8 bytes a step
        const int h = e & 1, l = (e >> 1) & 63, piece = e >> 7;
        const int t0 = piece / chunks * 32, d0 = piece % chunks * 32;
        int lowest = t0 + token_in_piece<KEYS>(l, h, 0), highest = t0 + token_in_piece<KEYS>(l, h, 7);
        if (lowest >= pg.to || (highest < pg.from && !grown)) continue;
        uint2 *at = reinterpret_cast<uint2 *>(codes + piece * 1024 + l * 16 + h * 8);
        uint2 had = make_uint2(0x80808080u, 0x80808080u);
        if (lowest < pg.from || highest >= pg.to) had = *at;
        uint32_t w[2] = {had.x, had.y};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int tok = t0 + token_in_piece<KEYS>(l, h, j), d = d0 + dim_in_piece<KEYS>(l, h, j);
            int code = (int)((w[j >> 2] >> (8 * (j & 3))) & 255) - 128;
            if (tok < pg.from) code = grown ? (int)rintf((float)code * again) : code;
            else if (tok < pg.to) code = d < dim ? code_of(value(tok, d), inv) : 0;
            w[j >> 2] = (w[j >> 2] & ~(255u << (8 * (j & 3)))) | (uint32_t)((code + 128) & 255) << (8 * (j & 3));
        }
        *at = make_uint2(w[0], w[1]);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(cmpq_kv_cache c, cmpq_kv_rows r, cmpq_heads K, cmpq_heads V,
                                                          cmpq_rotation rot, int32_t *status) {
    __shared__ float scratch[kThreads / 64];
    const Page pg = find_page(r, c.page, blockIdx.x, looks_over() ? status : nullptr);
    if (pg.seq < 0) return;
    const int64_t id = r.page_table[pg.seq * r.ld_table + pg.begin / c.page];
    if (id < 0 || id >= c.n_pages) {
        if (threadIdx.x == 0 && status) atomicOr(status, CMPQ_STATUS_RANGE);
        return;
    }
    if (blockIdx.z == 0) append_page<T, true>(c, pg, id, blockIdx.y, K, rot, status, scratch);
    else append_page<T, false>(c, pg, id, blockIdx.y, V, rot, status, scratch);
}

template <typename T, bool KEYS>
__device__ void read_page(const cmpq_kv_cache &c, const Page &pg, int64_t id, int head, const cmpq_heads &out) {
    const int dim = c.head_dim, chunks = (dim + 31) / 32, n = pg.to - pg.from;
    const uint8_t *codes = (KEYS ? c.k_codes : c.v_codes) + (id * c.kv_heads + head) * (int64_t)(c.page * chunks * 32);
    const float scale = (KEYS ? c.k_scale : c.v_scale)[id * c.kv_heads + head];
    T *base = static_cast<T *>(out.ptr) + head * out.head_stride;
    for (int e = threadIdx.x; e < n * dim; e += kThreads) {
        const int tok = pg.from + e / dim, d = e % dim, t = tok % 32, x = d % 32;
        const int byte = KEYS ? (x >> 3) * 256 + (t & 15) * 16 + (t >> 4) * 8 + (x & 7)
                              : ((t & 15) >> 2) * 256 + (x & 15) * 16 + (x >> 4) * 8 + (t >> 4) * 4 + (t & 3);
        const int code = (int)codes[(tok / 32 * chunks + d / 32) * 1024 + byte] - 128;
        base[(pg.row0 + pg.begin + tok - pg.first) * out.row_stride + d] = (T)((float)code * scale);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void read_kernel(cmpq_kv_cache c, cmpq_kv_rows r, cmpq_heads K, cmpq_heads V,
                                                        int32_t *status) {
    const Page pg = find_page(r, c.page, blockIdx.x, looks_over() ? status : nullptr);
    if (pg.seq < 0) return;
    const int64_t id = r.page_table[pg.seq * r.ld_table + pg.begin / c.page];
    if (id < 0 || id >= c.n_pages) {
        if (threadIdx.x == 0 && status) atomicOr(status, CMPQ_STATUS_RANGE);
        return;
    }
    if (blockIdx.z == 0) read_page<T, true>(c, pg, id, blockIdx.y, K);
    else read_page<T, false>(c, pg, id, blockIdx.y, V);
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

}  // namespace

extern "C" size_t cmpq_kv_page_bytes(int head_dim, int page) {
    if (head_dim < 1 || head_dim > 256 || page < 32 || page > 1024 || page % 32) return 0;
    return (size_t)page * 32 * ((head_dim + 31) / 32);
}

extern "C" int cmpq_kv_append(const cmpq_kv_cache *cache, const cmpq_kv_rows *rows, const cmpq_heads *K,
                              const cmpq_heads *V, int dtype, const cmpq_rotation *rotation, int32_t *status,
                              void *stream) {
    if (int rc = check_rows(cache, rows, K, V, dtype)) return rc;
    if (int rc = check_rotation(rotation, cache->head_dim)) return rc;
    if (rows->n_seq == 0 || rows->n_rows == 0 || rows->ld_table == 0) return CMPQ_OK;
    const cmpq_rotation rot = rotation ? *rotation : cmpq_rotation{};
    const dim3 grid = page_grid(*cache, *rows);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == CMPQ_F16) append_kernel<_Float16><<<grid, kThreads, 0, st>>>(*cache, *rows, *K, *V, rot, status);
    else if (dtype == CMPQ_BF16) append_kernel<__bf16><<<grid, kThreads, 0, st>>>(*cache, *rows, *K, *V, rot, status);
    else append_kernel<float><<<grid, kThreads, 0, st>>>(*cache, *rows, *K, *V, rot, status);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}

extern "C" int cmpq_kv_read(const cmpq_kv_cache *cache, const cmpq_kv_rows *rows, const cmpq_heads *K,
                            const cmpq_heads *V, int dtype, int32_t *status, void *stream) {
    if (int rc = check_rows(cache, rows, K, V, dtype)) return rc;
    if (rows->n_seq == 0 || rows->n_rows == 0 || rows->ld_table == 0) return CMPQ_OK;
    const dim3 grid = page_grid(*cache, *rows);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == CMPQ_F16) read_kernel<_Float16><<<grid, kThreads, 0, st>>>(*cache, *rows, *K, *V, status);
    else if (dtype == CMPQ_BF16) read_kernel<__bf16><<<grid, kThreads, 0, st>>>(*cache, *rows, *K, *V, status);
    else read_kernel<float><<<grid, kThreads, 0, st>>>(*cache, *rows, *K, *V, status);
    CMPQ_LAUNCH_CHECK();
    return CMPQ_OK;
}
