// kvs_evict_paged: a request's rows that received most attention, copied to pages of their own.
//
// Three launches.  keys: every row's mass, added up over the KV heads, as an order-preserving 32-bit key; protected rows get the
// largest.  select: a workgroup a request finds the m-th largest key by four passes of eight bits, then writes the list of the kept
// rows, ascending, ties to the lower index.  move: the rows' K, V and mass.
#include "paged.h"

namespace kvs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / kWave;

struct Kept { int m, first, recent; };      // rows kept, protected ones among them

__device__ __forceinline__ Kept kept_of(const Paged &pg, const int32_t *keep, int max_keep, int n_first, int n_recent, int b, int len)
{
    Kept k;
    k.m = min(len, min(max(keep[b], 0), max_keep));
    k.first = min(n_first, k.m);
    k.recent = min(n_recent, k.m - k.first);
    return k;
}

__global__ __launch_bounds__(kThreads) void evict_keys_kernel(const Paged pg, int n_kv_heads, const int32_t *__restrict__ keep, int max_keep, int n_first, int n_recent,
                                                              const float *__restrict__ mass, int64_t mass_stride, uint32_t *__restrict__ keys)
{
    const int b = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int len = len_of(pg, b);
    if (i >= len) return;
    const Kept k = kept_of(pg, keep, max_keep, n_first, n_recent, b, len);
    float sum = mass[(int64_t)b * n_kv_heads * mass_stride + i];
    for (int g = 1; g < n_kv_heads; ++g) sum += mass[((int64_t)b * n_kv_heads + g) * mass_stride + i];
    const uint32_t key = i < k.first || i >= len - k.recent ? 0xffffffffu : sum == sum ? score_key(sum) : 0u;
    keys[(int64_t)b * pg.max_ctx + i] = key;
}

// exclusive sum over the workgroup, and the total
__device__ __forceinline__ int scan_exclusive(int x, int *sums, int &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = x;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int y = __shfl_up(upto, s);
        upto += lane >= s ? y : 0;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + upto - x;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(const Paged pg, const int32_t *keep, int max_keep, int n_first, int n_recent, const uint32_t *__restrict__ keys,
                                                                   int32_t *__restrict__ list, int32_t *__restrict__ counts, int32_t *__restrict__ kept, int32_t *new_len)
{
    __shared__ int hist[256];
    __shared__ int sums[kSelWaves];
    __shared__ uint32_t found[2];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int len = len_of(pg, b);
    const int m = kept_of(pg, keep, max_keep, n_first, n_recent, b, len).m;
    const uint32_t *key = keys + (int64_t)b * pg.max_ctx;
    list += (int64_t)b * pg.max_ctx;
    __syncthreads();                                         // new_len may be the lengths
    if (tid == 0) {
        counts[b] = m;
        if (new_len) new_len[b] = m;
    }
    if (m == 0) return;
    uint32_t prefix = 0;                                     // the threshold's leading bits
    int want = m;                                            // ... and how many keys that begin with them are still to be taken
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < len; i += kSelThreads) {
            const uint32_t k = key[i];
            if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        const int mine = tid < 256 ? hist[255 - tid] : 0;    // from the largest digit down
        int total;
        const int before = scan_exclusive(mine, sums, total);
        if (before < want && before + mine >= want) {
            found[0] = (prefix << 8) | (uint32_t)(255 - tid);
            found[1] = (uint32_t)(want - before);
        }
        __syncthreads();
        prefix = found[0];
        want = (int)found[1];
    }
    // keys above the threshold, and the first `want` that equal it
    int taken = 0, equal = 0;
    for (int i0 = 0; i0 < len; i0 += kSelThreads) {
        const int i = i0 + tid;
        const uint32_t k = i < len ? key[i] : 0u;
        const bool above = i < len && k > prefix, same = i < len && k == prefix;
        int total;
        const int before = scan_exclusive((above ? 1 : 0) | (same ? 0x10000 : 0), sums, total);
        const int same_before = equal + (before >> 16);
        if (above || (same && same_before < want)) {
            const int at = taken + (before & 0xffff) + min(same_before, want);
            list[at] = i;
            if (kept) kept[(int64_t)b * max_keep + at] = i;
        }
        taken += total & 0xffff;
        equal += total >> 16;
    }
}

// PPL: 16-byte pieces of a row a lane moves, ROWS: rows of a wave
template <int PPL, int ROWS>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(const Paged pg, int n_kv_heads, int pieces_per_row, const int32_t *__restrict__ list, const int32_t *__restrict__ counts,
                                                              const int32_t *__restrict__ new_table, int new_width, uint4 *k_pool, uint4 *v_pool,
                                                              const float *__restrict__ mass, int64_t mass_stride, float *__restrict__ new_mass, int max_keep)
{
    const int b = blockIdx.y, lane = threadIdx.x & 63;
    const int64_t j0 = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * ROWS;
    const int m = counts[b];
    if (j0 >= m) return;
    list += (int64_t)b * pg.max_ctx;
    Paged to = pg;
    to.table = new_table;
    to.width = new_width;
    int64_t from_row[ROWS], to_row[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int j = (int)j0 + r;
        const int i = list[min(j, m - 1)];
        const int from = granule_of(pg, b, i / kGranule), into = new_table && j < m ? granule_of(to, b, j / kGranule) : -1;
        from_row[r] = from < 0 ? -1 : (int64_t)from * kGranule + i % kGranule;
        to_row[r] = into < 0 ? -1 : (int64_t)into * kGranule + j % kGranule;
        if (new_mass && j < m && lane < n_kv_heads) new_mass[((int64_t)b * n_kv_heads + lane) * max_keep + j] = mass[((int64_t)b * n_kv_heads + lane) * mass_stride + i];
    }
    uint4 kv[ROWS][PPL], vv[ROWS][PPL];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < PPL; ++i) {
            const int piece = lane + i * kWave;
            if (from_row[r] >= 0 && to_row[r] >= 0 && piece < pieces_per_row) {
                kv[r][i] = k_pool[from_row[r] * pieces_per_row + piece];
                vv[r][i] = v_pool[from_row[r] * pieces_per_row + piece];
            }
        }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < PPL; ++i) {
            const int piece = lane + i * kWave;
            if (from_row[r] >= 0 && to_row[r] >= 0 && piece < pieces_per_row) {
                k_pool[to_row[r] * pieces_per_row + piece] = kv[r][i];
                v_pool[to_row[r] * pieces_per_row + piece] = vv[r][i];
            }
        }
}

} // namespace

size_t evict_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx)
{
    if (check_shape(shape) != KVS_OK || batch <= 0 || max_ctx <= 0) return 256;
    return (((size_t)batch * 4 + (size_t)batch * (size_t)max_ctx * 8) + 511) / 256 * 256;
}

} // namespace kvs

extern "C" kvs_status kvs_evict_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                      const int32_t *keep, int64_t max_keep, int32_t n_first, int32_t n_recent, const float *mass, int64_t mass_stride,
                                      const int32_t *new_table, int32_t new_width, int32_t *kept, int32_t *new_len, float *new_mass,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace kvs;
    const char *me = "kvs_evict_paged";
    Paged pg;
    kvs_status st = check_paged(me, shape, cache, pages, &pg);
    if (st != KVS_OK) return st;
    if (max_keep < 0 || max_keep > 0x7fffff00LL) return fail(KVS_EINVAL, "%s: max_keep %lld", me, (long long)max_keep);
    if (n_first < 0 || n_recent < 0) return fail(KVS_EINVAL, "%s: a negative number of protected rows", me);
    if (new_table && (new_width < 0 || (int64_t)new_width * cache->page < max_keep))
        return fail(KVS_EINVAL, "%s: %d pages of %d rows do not hold %lld", me, new_width, cache->page, (long long)max_keep);
    if (mass_stride < pages->max_ctx) return fail(KVS_EINVAL, "%s: a mass stride of %lld for contexts of up to %lld", me, (long long)mass_stride, (long long)pages->max_ctx);
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(KVS_EINVAL, "%s: workspace must be 256-byte aligned", me);
    if (pages->batch == 0) return KVS_OK;
    if (!keep || !mass) return fail(KVS_EINVAL, "%s: keep or mass is NULL", me);
    if (pages->batch > 65535) return fail(KVS_EINVAL, "%s: %d requests in one call", me, pages->batch);
    if (mass == new_mass) return fail(KVS_EINVAL, "%s: new_mass may not be mass", me);
    if (!workspace || workspace_bytes < evict_paged_workspace_bytes(shape, pages->batch, pg.max_ctx)) return fail(KVS_EWORKSPACE, "%s: workspace too small", me);
    hipStream_t hs = (hipStream_t)stream;
    const int64_t stride = pg.max_ctx;
    uint32_t *keys = (uint32_t *)workspace;
    int32_t *list = (int32_t *)(keys + (int64_t)pg.batch * stride);
    int32_t *counts = list + (int64_t)pg.batch * stride;
    if (stride > 0) {
        hipLaunchKernelGGL(evict_keys_kernel, dim3((unsigned)((stride + kThreads - 1) / kThreads), (unsigned)pg.batch), dim3(kThreads), 0, hs, pg, shape->n_kv_heads, keep, (int)max_keep,
                           n_first, n_recent, mass, mass_stride, keys);
        if ((st = check_launch(me)) != KVS_OK) return st;
    }
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)pg.batch), dim3(kSelThreads), 0, hs, pg, keep, (int)max_keep, n_first, n_recent, keys, list, counts, kept, new_len);
    if ((st = check_launch(me)) != KVS_OK) return st;
    if (max_keep == 0 || stride == 0 || (!new_table && !new_mass)) return KVS_OK;
    const int ppr = (int)(shape->n_kv_heads * shape->head_dim * (int64_t)elem_bytes(shape->dtype) / 16);
    const int ppl = (ppr + kWave - 1) / kWave;
    const int64_t most = max_keep < stride ? max_keep : stride;
#define KVS_MOVE(P, R)                                                                                                                            \
    hipLaunchKernelGGL((evict_move_kernel<P, R>), dim3((unsigned)((most + (R) * kWaves - 1) / ((R) * kWaves)), (unsigned)pg.batch), dim3(kThreads), 0, hs, pg, \
                       shape->n_kv_heads, ppr, list, counts, new_table, new_width, (uint4 *)cache->k, (uint4 *)cache->v, mass, mass_stride, new_mass, (int)max_keep)
    if (ppl <= 1) KVS_MOVE(1, 4);
    else if (ppl <= 2) KVS_MOVE(2, 4);
    else if (ppl <= 4) KVS_MOVE(4, 2);
    else if (ppl <= 8) KVS_MOVE(8, 1);
    else if (ppl <= 16) KVS_MOVE(16, 1);
    else KVS_MOVE(32, 1);
#undef KVS_MOVE
    return check_launch(me);
}
