// kvs_store_paged: rows of K and V into the pages of their requests.
//
// A copy whose bytes bound it where it is large, and a chain of dependent trips to memory where it is small: the token's request,
// its position, its page.  A wave takes 4 KiB or so of rows and asks for their data first, so that only the stores wait for the
// chain.  (8192 rows of 8 heads of bf16, 128 channels, K and V: 67 MB in 11.9 us, 5.6 TB/s; one row of 4 heads 2.1 us, a launch and the chain.)
#include "paged.h"

namespace kvs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// The request that token s belongs to: how many end at or before it.  64 a step; the same for all lanes.
__device__ __forceinline__ int request_of_token(const Paged &pg, int s)
{
    if (!pg.cu_new) return s;
    const int lane = threadIdx.x & 63;
    int b = 0;
    for (int b0 = 0; b0 < pg.batch; b0 += 64) {
        const bool ended = b0 + lane < pg.batch && pg.cu_new[b0 + lane + 1] <= s;
        const int n = __popcll(__ballot(ended));
        b += n;
        if (n < 64) break;
    }
    return b;
}

// PPL: 16-byte pieces of a row a lane moves, ROWS: rows of a wave
template <int PPL, int ROWS>
__global__ __launch_bounds__(kThreads) void store_paged_kernel(const Paged pg, int pieces_per_row, int n_kv_heads, const uint4 *__restrict__ k_new, const uint4 *__restrict__ v_new,
                                                               uint4 *__restrict__ k_pool, uint4 *__restrict__ v_pool, float *__restrict__ mass, int64_t mass_stride)
{
    const int lane = threadIdx.x & 63;
    const int64_t s0 = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * ROWS;
    if (s0 >= pg.n_new) return;
    uint4 kv[ROWS][PPL], vv[ROWS][PPL];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t s = min(s0 + r, (int64_t)pg.n_new - 1);
#pragma unroll
        for (int i = 0; i < PPL; ++i) {
            const int pc = min(lane + i * kWave, pieces_per_row - 1);
            kv[r][i] = stream_load16(k_new + s * pieces_per_row + pc);
            vv[r][i] = stream_load16(v_new + s * pieces_per_row + pc);
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int s = (int)s0 + r;
        if (s >= pg.n_new) break;
        const int b = __builtin_amdgcn_readfirstlane(request_of_token(pg, s));
        if (b >= pg.batch) break;
        int lo, n;
        tokens_of(pg, b, lo, n);
        if (s < lo || s >= lo + n) continue;                   // a token of no request
        const int end = end_of(pg, b), len = min(end, pg.max_ctx);
        const int p = pg.sel_pos ? pg.sel_pos[s] : end - n + (s - lo);
        if (p < 0 || p >= len) continue;
        if (pg.sel_pos && s + 1 < lo + n && pg.sel_pos[s + 1] == p) continue;      // the last one counts
        const int at = granule_of(pg, b, p / kGranule);
        if (at >= 0) {
            const int64_t row = (int64_t)at * kGranule + p % kGranule;
#pragma unroll
            for (int i = 0; i < PPL; ++i) {
                const int piece = lane + i * kWave;
                if (piece < pieces_per_row) {
                    k_pool[row * pieces_per_row + piece] = kv[r][i];
                    v_pool[row * pieces_per_row + piece] = vv[r][i];
                }
            }
            if (mass && lane < n_kv_heads) mass[((int64_t)b * n_kv_heads + lane) * mass_stride + p] = 0.f;
        }
    }
}

} // namespace
} // namespace kvs

extern "C" kvs_status kvs_store_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                      const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new,
                                      const void *k_new, const void *v_new, float *mass, int64_t mass_stride, void *stream)
{
    using namespace kvs;
    const char *me = "kvs_store_paged";
    Paged pg;
    kvs_status st = check_paged(me, shape, cache, pages, &pg);
    if (st != KVS_OK || (st = check_new_tokens(me, shape, pages, cu_new, sel_pos, n_new, 0, 0, &pg)) != KVS_OK) return st;
    if (mass && mass_stride < pages->max_ctx) return fail(KVS_EINVAL, "%s: a mass stride of %lld for contexts of up to %lld", me, (long long)mass_stride, (long long)pages->max_ctx);
    if (n_new == 0 || pages->batch == 0) return KVS_OK;
    if (!k_new || !v_new) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    if (!aligned16(k_new) || !aligned16(v_new)) return fail(KVS_EINVAL, "%s: K/V pointers must be 16-byte aligned", me);
    const size_t pool = pool_bytes(shape, cache), rows = (size_t)n_new * shape->n_kv_heads * shape->head_dim * elem_bytes(shape->dtype), batch = (size_t)pages->batch;
    const size_t masses = batch * shape->n_kv_heads * (size_t)mass_stride * sizeof(float);
    st = check_apart(me, {{cache->k, pool, "the cache's K"}, {cache->v, pool, "the cache's V"}, {mass, masses, "mass"}},
                     {{k_new, rows, "k_new"}, {v_new, rows, "v_new"}, {pages->table, batch * pages->width * 4, "the page table"}, {pages->ctx_len, batch * 4, "ctx_len"},
                      {cu_new, (batch + 1) * 4, "cu_new"}, {sel_pos, (size_t)n_new * 4, "sel_pos"}});
    if (st == KVS_OK) st = check_apart(me, {{mass, masses, "mass"}}, {{cache->k, pool, "the cache's K"}, {cache->v, pool, "the cache's V"}});
    if (st != KVS_OK) return st;
    const int ppr = (int)(shape->n_kv_heads * shape->head_dim * (int64_t)elem_bytes(shape->dtype) / 16);
    const int ppl = (ppr + kWave - 1) / kWave;
#define KVS_STORE(P, R)                                                                                                                       \
    do {                                                                                                                                      \
        const int64_t blocks = ((n_new + (R) - 1) / (R) + kWaves - 1) / kWaves;                                                               \
        if (blocks > kMostWgs) return fail(KVS_EINVAL, "%s: too many rows", me);                                                              \
        hipLaunchKernelGGL((store_paged_kernel<P, R>), dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, pg, ppr,               \
                           shape->n_kv_heads, (const uint4 *)k_new, (const uint4 *)v_new, (uint4 *)cache->k, (uint4 *)cache->v, mass, mass_stride); \
    } while (0)
    if (ppl <= 1) KVS_STORE(1, 4);
    else if (ppl <= 2) KVS_STORE(2, 2);
    else if (ppl <= 4) KVS_STORE(4, 1);
    else if (ppl <= 8) KVS_STORE(8, 1);
    else if (ppl <= 16) KVS_STORE(16, 1);
    else KVS_STORE(32, 1);
#undef KVS_STORE
    return check_launch(me);
}
