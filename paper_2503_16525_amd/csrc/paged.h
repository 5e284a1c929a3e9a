// What the kernels over a cache in pages share (not part of the ABI).
#pragma once

#include "kvs_internal.h"

#include <initializer_list>

namespace kvs {

// A call's requests as its kernels see them.  Lengths, offsets, positions and page ids come from device memory and are not
// trusted: whatever stands there, every access stays inside the tensors that the host was told about.
struct Paged {
    const int32_t *table, *ctx_len, *cu_new, *sel_pos;
    int32_t batch, width, n_new;
    int32_t max_ctx;              // at most width pages of rows
    int32_t n_pages, page_log2;
    int32_t window, n_first;      // window 0: none
};

constexpr int kGranule = 16;      // rows that lie together whatever the page size: no page is shorter

kvs_status check_paged(const char *me, const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages, Paged *out);
// the same with a call's new tokens
kvs_status check_new_tokens(const char *me, const kvs_shape *shape, const kvs_page_table *pages, const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new,
                            int32_t window, int32_t n_first, Paged *out);
inline bool overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes)
{
    return (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}
// What a call writes may lie over nothing that it reads.  (NULL and nothing overlap nothing.)
struct Span { const void *at; size_t bytes; const char *name; };
inline kvs_status check_apart(const char *me, std::initializer_list<Span> written, std::initializer_list<Span> read)
{
    for (const Span &w : written)
        for (const Span &r : read)
            if (w.at && r.at && w.bytes && r.bytes && overlap(w.at, w.bytes, r.at, r.bytes)) return fail(KVS_EINVAL, "%s: %s overlaps %s", me, w.name, r.name);
    return KVS_OK;
}
inline size_t pool_bytes(const kvs_shape *shape, const kvs_paged_cache *c) { return (size_t)c->n_pages * c->page * shape->n_kv_heads * shape->head_dim * elem_bytes(shape->dtype); }
size_t attention_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx, int64_t n_new);
size_t mass_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx, int64_t n_new);
size_t evict_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx);

__device__ __forceinline__ int end_of(const Paged &pg, int b) { return max(pg.ctx_len[b], 0); }        // where new tokens end
__device__ __forceinline__ int len_of(const Paged &pg, int b) { return min(end_of(pg, b), pg.max_ctx); } // rows that are taken

// The tokens of request b: [lo, lo + n) of the call's.
__device__ __forceinline__ void tokens_of(const Paged &pg, int b, int &lo, int &n)
{
    if (!pg.cu_new) { lo = b; n = 1; return; }
    lo = min(max(pg.cu_new[b], 0), pg.n_new);
    n = min(max(pg.cu_new[b + 1], lo), pg.n_new) - lo;
}

// Position of token i of a request's n, -1 where it sees nothing, at most the last that is taken.  (Of a context that is longer than was
// promised the last tokens stand behind that, not in the place of rows that are there.)
__device__ __forceinline__ int position_of(const Paged &pg, int lo, int n, int i, int len, int end)
{
    const int p = pg.sel_pos ? pg.sel_pos[lo + i] : end - n + i;
    return p < 0 ? -1 : min(p, len - 1);
}

// Which 16 rows of the pool rows 16 gi .. 16 gi + 15 of request b are, -1: none.
__device__ __forceinline__ int granule_of(const Paged &pg, int b, int gi)
{
    const int shift = pg.page_log2 - 4, at = gi >> shift;
    if (gi < 0 || at >= pg.width) return -1;
    const int id = pg.table[(int64_t)b * pg.width + at];
    return (uint32_t)id < (uint32_t)pg.n_pages ? (id << shift) + (gi & ((1 << shift) - 1)) : -1;
}

// A call's rows (tokens times the query heads that share a KV head) in blocks of R rows, none of which holds two requests: which request
// block u belongs to, which of its blocks it is, the request's tokens [tok0, tok0 + n_tok), context length and end.  All lanes of a wave ask
// for the same block; 64 requests a step, whose offsets and lengths come in one trip to memory.
struct Block { int b, blk, tok0, n_tok, len, end; };
template <int R>
__device__ __forceinline__ bool find_block(const Paged &pg, int grp, int u, Block &out)
{
    if (!pg.cu_new) {
        const int per = (grp + R - 1) / R, b = u / per;
        if (b >= pg.batch) return false;
        const int end = end_of(pg, b);
        out = {b, u - b * per, b, 1, min(end, pg.max_ctx), end};
        return true;
    }
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < pg.batch; b0 += 64) {
        int lo = 0, n = 0, end = 0;
        if (b0 + lane < pg.batch) {
            end = end_of(pg, b0 + lane);
            tokens_of(pg, b0 + lane, lo, n);
        }
        const int mine = (n * grp + R - 1) / R;
        int upto = mine;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int x = __shfl_up(upto, s);
            upto += lane >= s ? x : 0;
        }
        const unsigned long long past = __ballot(base + upto > u);
        if (past) {
            const int at = __ffsll((long long)past) - 1;
            end = __builtin_amdgcn_readlane(end, at);
            out = {b0 + at, u - base - __builtin_amdgcn_readlane(upto - mine, at), __builtin_amdgcn_readlane(lo, at), __builtin_amdgcn_readlane(n, at), min(end, pg.max_ctx), end};
            return true;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// How many such blocks there can be, whatever the offsets.
inline int64_t most_blocks(const Paged &pg, int grp, int r)
{
    if (!pg.cu_new) return (int64_t)pg.batch * ((grp + r - 1) / r);
    const int64_t rows = (int64_t)pg.n_new * grp, reqs = pg.batch < pg.n_new ? pg.batch : pg.n_new;
    return (rows + reqs * (r - 1)) / r;
}

} // namespace kvs
