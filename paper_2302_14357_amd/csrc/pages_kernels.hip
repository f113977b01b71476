// Page tables, lengths and partly filled pages follow the chosen hypotheses.
#include "op_device.h"

// 16 bytes on any element's boundary
typedef unsigned pages_piece __attribute__((ext_vector_type(4), aligned(2)));

struct PagesP {
    const int *parents, *tables, *lens;
    const uint8_t *finished;
    int *out_tables, *out_lens, *status;
    int64_t ld, ld_out;
    int64_t cp, ct, ch;   // bytes from page to page, token to token, head to head
    int beams, width, pages, page, heads, head_bytes, appended, shares;
    bool flat;   // a page's tokens are one run of bytes
    char *caches[TBS_MAX_CACHES];
};

// One launch: a workgroup a row, cache and share of the page.  Each works out its group's places by itself (beams <= 32: a wave, a
// lane a place), which is less than a second launch would cost; those of a row that copies nothing leave then.
__global__ void __launch_bounds__(256)
k_pages_reorder(PagesP p) {
    const int N = p.beams, row = blockIdx.x, c = row % N, r0 = row - c, lane = threadIdx.x & 63;
    const bool writer = blockIdx.y == 0 && blockIdx.z == 0;
    // every wave does the same
    int parent = -1, was = 0, len = 0, whole_l = 0;   // of place `lane`; tokens of row `lane` before and now, and how many pages at its table's head others may name too
    if (lane < N) {
        parent = p.parents[r0 + lane];
        if ((unsigned)parent >= (unsigned)N) parent = -1;
        was = p.lens[r0 + lane];
        len = was >= 0 ? min(was, p.width * p.page - p.appended) + p.appended : min(~was, p.width * p.page);   // (no more than a table holds)
        whole_l = was == -1 ? p.width : len / p.page;   // (a row without a hypothesis has had one perhaps, or a dropped one's place: any of its pages may be shared)
    }
    if (__shfl(was, max(parent, 0)) == -1) parent = -1;   // (nothing to go on from: its children are places without a hypothesis as well)
    bool first = parent >= 0;
    unsigned has_child = 0;
    for (int i = 0; i < N; ++i) {
        const int q = __shfl(parent, i);
        if (i < lane && q == parent) first = false;
        if (q >= 0) has_child |= 1u << q;
    }
    unsigned left = ~has_child & (N == 32 ? ~0u : (1u << N) - 1);                  // rows without children
    const unsigned need = (unsigned)__ballot(lane < N && !first);                  // places that take the own pages of one
    const int mine = __shfl(parent, c), is_first = (need >> c & 1) == 0;
    for (int k = __popc(need & ((1u << c) - 1)); k > 0; --k) left &= left - 1;
    const int giver = is_first ? mine : __ffs(left) - 1;
    const int L = mine >= 0 ? __shfl(len, max(mine, 0)) : 0, full = L / p.page;
    // The giver's own pages begin behind its whole ones.  Where it has more of these than the child keeps of its parent's, those in between are free only if
    // the giver alone names them.  (Columns to lanes, rows to waves.  A first step of 64 groups of eight with tables of 256 pages, 24 caches, one
    // hypothesis a group: 42 us, 25 where all have tokens.)
    const int given = __shfl(whole_l, giver);
    bool drop = false;
    if (mine >= 0 && !is_first && given > full) {   // (the same for the whole workgroup)
        int shared = 0;
        for (int col = full + lane; col < min(given, p.width); col += 64) {
            const int id = p.tables[(int64_t)(r0 + giver) * p.ld + col];   // (an entry that names no page is shared with nobody)
            for (int other = threadIdx.x >> 6; other < N; other += 4)
                shared |= other != giver && (unsigned)id < (unsigned)p.pages && p.tables[(int64_t)(r0 + other) * p.ld + col] == id;
        }
        drop = __syncthreads_or(shared);
    }
    const int *from = p.tables + (int64_t)(r0 + max(mine, 0)) * p.ld, *own = p.tables + (int64_t)(r0 + giver) * p.ld;
    if (writer) {
        const int whole = mine >= 0 && !drop ? full : 0;
        for (int i = threadIdx.x; i < p.width; i += 256) p.out_tables[(int64_t)row * p.ld_out + i] = i < whole ? from[i] : own[i];
        if (threadIdx.x == 0) {
            p.out_lens[row] = mine < 0 || drop ? -1 : p.finished && p.finished[row] ? ~L : L;
            if (drop && p.status) atomicAdd(p.status, 1);
        }
    }
    if (mine < 0 || is_first || drop || full >= p.width || L % p.page == 0) return;
    if (!p.caches[blockIdx.y]) return;
    const int src = from[full], dst = own[full];
    if ((unsigned)src >= (unsigned)p.pages || (unsigned)dst >= (unsigned)p.pages || src == dst) return;
    char *cache = p.caches[blockIdx.y];
    const char *x = cache + src * p.cp;
    char *y = cache + dst * p.cp;
    const int tid = (int)(blockIdx.z * 256 + threadIdx.x), threads = p.shares * 256;
    auto tail = [&](int64_t at, int n) {
        for (int j = 0; j < n; j += 2) *(uint16_t *)(y + at + j) = *(const uint16_t *)(x + at + j);
    };
    if (p.flat) {
        // the page's first tokens are one run of bytes, four pieces of 16 a thread on their way at a time (bound by memory: 512 rows, half of them copying 31 to
        // 59 tokens of 2 KB in 24 caches, 178 us, 4.7 TB/s read and written; with stores that stay in the caches 187)
        const int64_t bytes = (int64_t)(L % p.page) * p.head_bytes, whole = bytes / 16;
        int64_t i = tid;
        for (; i + 3 * threads < whole; i += 4 * threads) {
            pages_piece u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) __builtin_memcpy(&u[k], x + (i + k * threads) * 16, 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) __builtin_nontemporal_store(u[k], (pages_piece *)(y + (i + k * threads) * 16));
        }
        for (; i < whole; i += threads) {
            uint4 u;
            __builtin_memcpy(&u, x + i * 16, 16);
            __builtin_memcpy(y + i * 16, &u, 16);
        }
        if (tid == 0) tail(whole * 16, (int)(bytes - whole * 16));
        return;
    }
    const unsigned pieces = (p.head_bytes + 15) / 16;
    const int64_t total = (int64_t)(L % p.page) * p.heads * pieces;
    for (int64_t i = tid; i < total; i += threads) {
        const int64_t h = total <= UINT32_MAX ? (unsigned)i / pieces : i / pieces;   // (a long division takes a hundred instructions)
        const int64_t t = total <= UINT32_MAX ? (unsigned)h / (unsigned)p.heads : h / p.heads;
        const int k = (int)(i - h * pieces), n = p.head_bytes - k * 16;
        const int64_t at = t * p.ct + (h - t * p.heads) * p.ch + k * 16;
        if (n >= 16) {
            uint4 u;
            __builtin_memcpy(&u, x + at, 16);
            __builtin_memcpy(y + at, &u, 16);
        } else {
            tail(at, n);
        }
    }
}

static bool pages_overlap(const void *a, int64_t na, const void *b, int64_t nb) {
    return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

extern "C" int tbs_beam_reorder(const tbs_beam_reorder_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_beam_reorder_args &a = *args;
    if (!op_dtype_known(a.dtype) || a.beams < 1 || a.beams > TBS_MAX_BEAM || a.rows < 0 || a.rows % a.beams || a.table_width < 1 || a.pages < 1 ||
        a.page < 1 || a.page > 65536 || (int64_t)a.table_width * a.page > (1 << 30) || a.n_caches < 0 || a.n_caches > TBS_MAX_CACHES ||
        (a.appended != 0 && a.appended != 1))
        return TBS_EINVAL;
    if (a.n_caches > 0) {
        if (!a.caches || a.kv_heads < 1 || a.kv_heads > 65535 || a.dim < 1 || a.dim > 65536) return TBS_EINVAL;
        const int64_t strides[] = {a.cache_page, a.cache_token, a.cache_head};
        for (int64_t s : strides)
            if (s < 0 || s > INT64_MAX / 64 / INT32_MAX) return TBS_EINVAL;
        if ((a.kv_heads > 1 && a.cache_head < a.dim) || (a.page > 1 && a.cache_token < a.dim) || (a.pages > 1 && a.cache_page < a.dim)) return TBS_EINVAL;
        for (int i = 0; i < a.n_caches; ++i)
            if (!a.caches[i] || (uintptr_t)a.caches[i] % op_dtype_size(a.dtype)) return TBS_EINVAL;
    }
    if (a.rows == 0) return TBS_OK;
    if (!a.parents || !a.tables || !a.lens || !a.out_tables || !a.out_lens || a.ld_tables < a.table_width || a.ld_out_tables < a.table_width)
        return TBS_EINVAL;
    if (pages_overlap(a.tables, ((a.rows - 1) * a.ld_tables + a.table_width) * 4, a.out_tables, ((a.rows - 1) * a.ld_out_tables + a.table_width) * 4) ||
        pages_overlap(a.lens, (int64_t)a.rows * 4, a.out_lens, (int64_t)a.rows * 4))
        return TBS_EINVAL;
    const int64_t es = (int64_t)op_dtype_size(a.dtype);
    PagesP p = {};
    p.parents = a.parents, p.tables = a.tables, p.lens = a.lens, p.finished = a.finished;
    p.out_tables = a.out_tables, p.out_lens = a.out_lens, p.status = a.status;
    p.ld = a.ld_tables, p.ld_out = a.ld_out_tables;
    p.cp = a.cache_page * es, p.ct = a.cache_token * es, p.ch = a.cache_head * es;
    p.beams = a.beams, p.width = a.table_width, p.pages = a.n_caches > 0 ? a.pages : INT32_MAX, p.page = a.page, p.heads = a.kv_heads, p.head_bytes = (int)(a.dim * es);
    p.appended = a.appended;
    if (a.n_caches > 0 && p.heads > 1 && p.ch == p.head_bytes && (int64_t)p.heads * p.head_bytes < INT32_MAX / 2) {   // a token's heads side by side: one row
        p.head_bytes *= p.heads;
        p.heads = 1;
    }
    p.flat = p.heads == 1 && p.ct == p.head_bytes;
    for (int i = 0; i < a.n_caches; ++i) p.caches[i] = (char *)a.caches[i];
    const int64_t units = (int64_t)a.rows * (a.n_caches > 0 ? a.n_caches : 1), page_bytes = (int64_t)a.page * p.heads * p.head_bytes;
    int64_t shares = 2048 / units, most = (page_bytes + 16383) / 16384;   // a share of 16 KB at least
    if (shares > most) shares = most;
    p.shares = shares < 1 ? 1 : (int)shares;
    const hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(k_pages_reorder, dim3(a.rows, a.n_caches > 0 ? a.n_caches : 1, p.shares), dim3(256), 0, st, p);
    return hipGetLastError() == hipSuccess ? TBS_OK : TBS_EHIP;
}
