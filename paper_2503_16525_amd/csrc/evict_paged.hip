// kvs_evict_paged: a request's rows that received most attention, copied to pages of their own.
//
// Every row has a 32-bit key, its mass added up over the KV heads, order-preserving; protected rows have the largest.  The m-th largest key
// is found by its digits, 11, 11 and 10 bits from the top: a count of the digit's values in LDS tells which one the key has.  Rows
// above it stay, and so many of those that equal it, from the lowest index on.
//   Up to kSmall rows a workgroup a request holds all keys in registers.  Longer contexts take three launches for it: segments make
//   their keys and count their first digits; parts add these up, set their keys of the one value aside and count the second
//   digits; a workgroup a request finds the rest among those; a fourth counts what stays of every 256 rows.
//   The last launch moves: a workgroup for every 256 rows ranks its own behind those before it and copies them.
// What bounds it: the copy, at most; the keys' passes are a few dependent trips to memory each.  (131072 rows of 4 heads to 65536: keys 4.8 us, first
// digits 7.5, the rest 6.2, counts 4.6, the copy of 268 MB 52, 5.1 TB/s, 86 with the launches' gaps; 4097 rows to 3584 8.3 and 7.5.)
#include "paged.h"

namespace kvs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kSub = kThreads;              // rows of a moving workgroup
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / kWave;
constexpr int kMostKeys = 16;                // of a thread
constexpr int kSmall = kSelThreads * kMostKeys;
constexpr int kSeg = 2048;                  // rows whose first digits are counted together
constexpr int kBins = 2048;                 // values of a digit
constexpr int kPart = 8192;                 // keys that a workgroup looks through

struct Picked { uint32_t key; int32_t want, m, len; };      // the m-th largest key, how many that equal it stay

// Keys of rows i0, i0 + kSelThreads, ..: all rows' masses of a few heads are asked for together, and added in the heads' order.
template <int N>
__device__ __forceinline__ void keys_of(uint32_t (&key)[N], const Paged &pg, int b, int i0, int len, int m, int n_first, int n_recent, int n_kv_heads, const float *__restrict__ mass, int64_t mass_stride)
{
    constexpr int HEADS = N <= 8 ? 4 : 2;
    const int first = min(n_first, m), recent = min(n_recent, m - first);
    const float *const from = mass + (int64_t)b * n_kv_heads * mass_stride;
    float sum[N];
    for (int g0 = 0; g0 < n_kv_heads; g0 += HEADS) {
        float x[HEADS][N];
#pragma unroll
        for (int h = 0; h < HEADS; ++h)
#pragma unroll
            for (int j = 0; j < N; ++j) x[h][j] = from[min(g0 + h, n_kv_heads - 1) * mass_stride + min((int64_t)i0 + j * kSelThreads, (int64_t)len - 1)];
#pragma unroll
        for (int h = 0; h < HEADS; ++h)
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] = g0 + h == 0 ? x[h][j] : g0 + h < n_kv_heads ? sum[j] + x[h][j] : sum[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int64_t i = (int64_t)i0 + j * kSelThreads;
        key[j] = i >= len ? 0u : i < first || i >= len - recent ? 0xffffffffu : sum[j] == sum[j] ? score_key(sum[j]) : 0u;
    }
}

__device__ __forceinline__ int kept_of(const int32_t *keep, int max_keep, int b, int len) { return min(len, min(max(keep[b], 0), max_keep)); }

// exclusive sum over the workgroup, and the total
template <int WAVES>
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
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + upto - x;
}

// From the counts of a digit's values: the value of the want-th largest, and how many of that value are still wanted.  Two values a thread.
__device__ __forceinline__ void find_digit(int large, int small, int *sums, int *found, uint32_t &digit, int &want)
{
    int total;
    const int before = scan_exclusive<kSelWaves>(large + small, sums, total);
    if (before < want && before + large >= want) { found[0] = kBins - 1 - 2 * (int)threadIdx.x; found[1] = want - before; }
    else if (before + large < want && before + large + small >= want) { found[0] = kBins - 2 - 2 * (int)threadIdx.x; found[1] = want - before - large; }
    __syncthreads();
    digit = (uint32_t)found[0];
    want = found[1];
    __syncthreads();
}

// Up to kSmall rows a request: keys, the m-th of them, and what stays of every kSub rows.  (One load after another a thread and eight keys at the most: 8192 rows
// 20.7 us with the copy, now 17.8; 16384 rows by four launches 34.8, now 28.6.)
// KPT: keys of a thread
template <int KPT>
__global__ __launch_bounds__(kSelThreads) void evict_small_kernel(const Paged pg, int n_kv_heads, const int32_t *keep, int max_keep, int n_first, int n_recent,
                                                                  const float *__restrict__ mass, int64_t mass_stride, uint32_t *__restrict__ keys, int64_t stride, Picked *__restrict__ picked,
                                                                  int2 *__restrict__ counts, int subs, int32_t *new_len)
{
    __shared__ int hist[kBins];
    __shared__ int sums[kSelWaves], found[2];
    __shared__ int above_s[(KPT * kSelThreads) / kSub], equal_s[(KPT * kSelThreads) / kSub];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int len = len_of(pg, b);
    const int m = kept_of(keep, max_keep, b, len);
    uint32_t key[KPT] = {};
    if (len > 0) keys_of(key, pg, b, tid, len, m, n_first, n_recent, n_kv_heads, mass, mass_stride);
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = tid + j * kSelThreads;
        if (i < len) keys[(int64_t)b * stride + i] = key[j];
    }
    if (tid < (KPT * kSelThreads) / kSub) above_s[tid] = equal_s[tid] = 0;
    uint32_t prefix = 0;
    int want = m;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t mask = pass == 2 ? 1023u : 2047u;
        hist[tid] = hist[tid + kSelThreads] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < KPT; ++j)
            if (tid + j * kSelThreads < len && (pass == 0 || key[j] >> (pass == 1 ? 21 : 10) == prefix)) atomicAdd(&hist[(key[j] >> shift) & mask], 1);
        __syncthreads();
        uint32_t digit = 0;
        if (m > 0) find_digit(hist[kBins - 1 - 2 * tid], hist[kBins - 2 - 2 * tid], sums, found, digit, want);
        prefix = (prefix << (pass == 2 ? 10 : 11)) | digit;
    }
    if (m == 0) { prefix = 0xffffffffu; want = 0; }
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = tid + j * kSelThreads;
        const int above = __popcll(__ballot(i < len && key[j] > prefix)), equal = __popcll(__ballot(i < len && key[j] == prefix));
        if (lane == 0) { atomicAdd(&above_s[i / kSub], above); atomicAdd(&equal_s[i / kSub], equal); }
    }
    __syncthreads();
    for (int i = tid; i < subs; i += kSelThreads) counts[(int64_t)b * subs + i] = make_int2(above_s[i], equal_s[i]);
    if (tid == 0) {
        picked[b] = {prefix, want, m, len};
        if (new_len) new_len[b] = m;
    }
}

__global__ __launch_bounds__(kSelThreads) void evict_keys_kernel(const Paged pg, int n_kv_heads, const int32_t *__restrict__ keep, int max_keep, int n_first, int n_recent,
                                                              const float *__restrict__ mass, int64_t mass_stride, uint32_t *__restrict__ keys, int64_t stride, uint32_t *__restrict__ firsts)
{
    __shared__ int hist[kBins];
    const int b = blockIdx.y, tid = threadIdx.x, lo = (int)blockIdx.x * kSeg;
    const int len = len_of(pg, b);
    if (lo >= len) return;
    const int m = kept_of(keep, max_keep, b, len);
#pragma unroll
    for (int j = 0; j < kBins / kSelThreads; ++j) hist[tid + j * kSelThreads] = 0;
    __syncthreads();
    uint32_t key[kSeg / kSelThreads];
    keys_of(key, pg, b, lo + tid, len, m, n_first, n_recent, n_kv_heads, mass, mass_stride);
#pragma unroll
    for (int j = 0; j < kSeg / kSelThreads; ++j) {
        const int64_t i = lo + tid + j * kSelThreads;
        if (i < len) {
            keys[(int64_t)b * stride + i] = key[j];
            atomicAdd(&hist[key[j] >> 21], 1);
        }
    }
    __syncthreads();
    uint32_t *to = firsts + ((int64_t)b * gridDim.x + blockIdx.x) * (kBins / 2);       // two counts of at most kSeg a word
    static_assert(kBins == 2 * kSelThreads, "a word a thread");
    to[tid] = (uint32_t)hist[2 * tid] | (uint32_t)hist[2 * tid + 1] << 16;
}

// The first digit of the m-th key, from all segments' counts; then, of a part of the keys, those that have it: set aside, and their second digits
// counted.  (One workgroup for all keys of a request issued instructions for 21 us of 131072.)
__global__ __launch_bounds__(kSelThreads) void evict_scan_kernel(const Paged pg, const int32_t *__restrict__ keep, int max_keep, const uint32_t *__restrict__ keys, int64_t stride,
                                                                 const uint32_t *__restrict__ firsts, int segs, uint32_t *__restrict__ aside, int32_t *__restrict__ n_aside,
                                                                 uint32_t *__restrict__ seconds, Picked *__restrict__ picked)
{
    __shared__ int hist[kBins];
    __shared__ int sums[kSelWaves], found[2], taken;
    const int b = blockIdx.y, part = blockIdx.x, parts = gridDim.x, tid = threadIdx.x;
    const int len = len_of(pg, b);
    const int m = kept_of(keep, max_keep, b, len);
    const int64_t lo = (int64_t)part * kPart;
    if (lo >= len || m == 0) return;
    uint32_t key[kPart / kSelThreads];
#pragma unroll
    for (int j = 0; j < kPart / kSelThreads; ++j) {
        const int64_t i = lo + j * kSelThreads + tid;
        key[j] = i < len ? keys[(int64_t)b * stride + i] : 0u;
    }
    const int live = (len + kSeg - 1) / kSeg;
    int large = 0, small = 0;                                // word kBins / 2 - 1 - tid
#pragma unroll 32
    for (int s = 0; s < live; ++s) {
        const uint32_t w = firsts[((int64_t)b * segs + s) * (kBins / 2) + kBins / 2 - 1 - tid];
        large += (int)(w >> 16);
        small += (int)(w & 0xffffu);
    }
    hist[tid] = hist[tid + kSelThreads] = 0;
    if (tid == 0) taken = 0;
    uint32_t digit;
    int want = m;
    find_digit(large, small, sums, found, digit, want);
    aside += (int64_t)b * stride + lo;
#pragma unroll
    for (int j = 0; j < kPart / kSelThreads; ++j) {
        const bool mine = lo + j * kSelThreads + tid < len && key[j] >> 21 == digit;
        const unsigned long long all = __ballot(mine);
        int at = 0;
        if ((tid & 63) == 0 && all) at = atomicAdd(&taken, __popcll(all));          // (any order: only their values count)
        at = __builtin_amdgcn_readfirstlane(at);
        if (mine) {
            atomicAdd(&hist[(key[j] >> 10) & 2047u], 1);
            aside[at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0u))] = key[j];
        }
    }
    __syncthreads();
    seconds[((int64_t)b * parts + part) * (kBins / 2) + tid] = (uint32_t)hist[2 * tid] | (uint32_t)hist[2 * tid + 1] << 16;
    if (tid == 0) {
        n_aside[(int64_t)b * parts + part] = taken;
        if (part == 0) picked[b] = {digit, want, m, len};    // so far
    }
}

// The second digit from all parts' counts, the third from the keys set aside that have both.
__global__ __launch_bounds__(kSelThreads) void evict_pick_kernel(const Paged pg, const int32_t *keep, int max_keep, int64_t stride, const uint32_t *__restrict__ aside, const int32_t *__restrict__ n_aside, const uint32_t *__restrict__ seconds, int parts, Picked *picked, int32_t *new_len)
{
    __shared__ int hist[kBins];
    __shared__ int sums[kSelWaves], found[2];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int len = len_of(pg, b);
    const int m = kept_of(keep, max_keep, b, len);
    uint32_t key = 0xffffffffu;
    int want = m;
    if (m > 0) {
        const int live = (int)(((int64_t)len + kPart - 1) / kPart);
        const Picked first = picked[b];
        // a wave a part; the first keys of its first one are asked for before it is known which count
        constexpr int EARLY = 8;
        const int wave = tid >> 6, lane = tid & 63;
        const uint32_t *const from = aside + (int64_t)b * stride;
        uint32_t early[EARLY];
        int n_early = 0;
        if (wave < live) {
            n_early = n_aside[(int64_t)b * parts + wave];
#pragma unroll
            for (int j = 0; j < EARLY; ++j) early[j] = from[min((int64_t)wave * kPart + j * kWave + lane, (int64_t)len - 1)];
        }
        int large = 0, small = 0;                            // word kBins / 2 - 1 - tid
#pragma unroll 16
        for (int s = 0; s < live; ++s) {
            const uint32_t w = seconds[((int64_t)b * parts + s) * (kBins / 2) + kBins / 2 - 1 - tid];
            large += (int)(w >> 16);
            small += (int)(w & 0xffffu);
        }
        uint32_t digit;
        want = first.want;
        find_digit(large, small, sums, found, digit, want);
        key = first.key << 11 | digit;
        hist[tid] = hist[tid + kSelThreads] = 0;
        __syncthreads();
        auto count = [&](uint32_t k) { if (k >> 10 == key) atomicAdd(&hist[k & 1023u], 1); };
#pragma unroll
        for (int j = 0; j < EARLY; ++j)
            if (j * kWave + lane < n_early) count(early[j]);
        for (int p = wave; p < live; p += kSelWaves) {
            const int n = p == wave ? n_early : n_aside[(int64_t)b * parts + p];
#pragma unroll 8
            for (int i = (p == wave ? EARLY * kWave : 0) + lane; i < n; i += kWave) count(from[(int64_t)p * kPart + i]);
        }
        __syncthreads();
        find_digit(hist[kBins - 1 - 2 * tid], hist[kBins - 2 - 2 * tid], sums, found, digit, want);
        key = key << 10 | digit;
    }
    if (tid == 0) {
        picked[b] = {key, want, m, len};
        if (new_len) new_len[b] = m;
    }
}

__global__ __launch_bounds__(kThreads) void evict_count_kernel(const uint32_t *__restrict__ keys, int64_t stride, const Picked *__restrict__ picked, int2 *__restrict__ counts, int subs)
{
    const int b = blockIdx.y, lane = threadIdx.x & 63;
    const int sub = (int)blockIdx.x * kWaves + (threadIdx.x >> 6);          // a wave for kSub rows
    const Picked p = picked[b];
    if (sub >= subs || (int64_t)sub * kSub >= p.len) return;
    int above = 0, equal = 0;
#pragma unroll
    for (int j = 0; j < kSub / kWave; ++j) {
        const int64_t i = (int64_t)sub * kSub + j * kWave + lane;
        const uint32_t k = i < p.len ? keys[(int64_t)b * stride + i] : 0u;
        above += __popcll(__ballot(i < p.len && k > p.key));
        equal += __popcll(__ballot(i < p.len && k == p.key));
    }
    if (lane == 0) counts[(int64_t)b * subs + sub] = make_int2(above, equal);
}

// PPL: 16-byte pieces of a row a lane moves, ROWS: rows of a wave at a time
template <int PPL, int ROWS>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(const Paged pg, int n_kv_heads, int pieces_per_row, const uint32_t *__restrict__ keys, int64_t stride,
                                                              const Picked *__restrict__ picked, const int2 *__restrict__ counts, int subs,
                                                              const int32_t *__restrict__ new_table, int new_width, uint4 *k_pool, uint4 *v_pool, const float *__restrict__ mass,
                                                              int64_t mass_stride, int32_t *__restrict__ kept, float *__restrict__ new_mass, int max_keep)
{
    __shared__ int sums[kWaves];
    __shared__ int4 move_s[kSub];                            // 16 rows of the pool each way, and the row among them
    const int b = blockIdx.y, sub = blockIdx.x, part = blockIdx.z, parts = gridDim.z, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Picked p = picked[b];
    const int64_t i = (int64_t)sub * kSub + tid;
    if ((int64_t)sub * kSub >= p.len || p.m == 0) return;
    const uint32_t key = i < p.len ? keys[(int64_t)b * stride + i] : 0u;
    int above = 0, equal = 0;                                // before the workgroup's rows
    for (int s = tid; s < sub; s += kThreads) {
        const int2 c = counts[(int64_t)b * subs + s];
        above += c.x;
        equal += c.y;
    }
    int total;
    scan_exclusive<kWaves>(above, sums, total);
    above = total;
    scan_exclusive<kWaves>(equal, sums, total);
    equal = total;
    const bool is_above = i < p.len && key > p.key, is_equal = i < p.len && key == p.key;
    const int before = scan_exclusive<kWaves>((is_above ? 1 : 0) | (is_equal ? 0x10000 : 0), sums, total);
    const int equal_before = equal + (before >> 16);
    const int first = above + min(equal, p.want);            // rank of the workgroup's first kept row
    const int n = above + (total & 0xffff) + min(equal + (total >> 16), p.want) - first;
    if (is_above || (is_equal && equal_before < p.want)) {
        const int rank = above + (before & 0xffff) + min(equal_before, p.want);
        if (kept && part == 0) kept[(int64_t)b * max_keep + rank] = (int)i;
        for (int g = part; new_mass && g < n_kv_heads; g += parts)
            new_mass[((int64_t)b * n_kv_heads + g) * max_keep + rank] = mass[((int64_t)b * n_kv_heads + g) * mass_stride + i];
        if (new_table) {
            Paged to = pg;
            to.table = new_table;
            to.width = new_width;
            const int from = granule_of(pg, b, (int)i / kGranule), into = granule_of(to, b, rank / kGranule);
            move_s[rank - first] = make_int4(max(from, 0), from < 0 ? -1 : into, (int)i % kGranule, rank % kGranule);
        }
    }
    if (!new_table) return;
    __syncthreads();
    for (int r0 = (part * kWaves + wave) * ROWS; r0 < n; r0 += parts * kWaves * ROWS) {
        uint4 kv[ROWS][PPL], vv[ROWS][PPL];
        int64_t to_row[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int4 mv = move_s[min(r0 + r, n - 1)];
            const int64_t from_row = (int64_t)mv.x * kGranule + mv.z;
            to_row[r] = r0 + r < n && mv.y >= 0 ? (int64_t)mv.y * kGranule + mv.w : -1;
#pragma unroll
            for (int u = 0; u < PPL; ++u) {
                const int piece = min(lane + u * kWave, pieces_per_row - 1);
                kv[r][u] = stream_load16(k_pool + from_row * pieces_per_row + piece);
                vv[r][u] = stream_load16(v_pool + from_row * pieces_per_row + piece);
            }
        }
        asm volatile("" ::: "memory");                       // all loads before the first store
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int u = 0; u < PPL; ++u) {
                const int piece = lane + u * kWave;
                if (to_row[r] >= 0 && piece < pieces_per_row) {
                    k_pool[to_row[r] * pieces_per_row + piece] = kv[r][u];
                    v_pool[to_row[r] * pieces_per_row + piece] = vv[r][u];
                }
            }
    }
}

struct Layout { int64_t stride, subs, segs, parts; size_t picked, counts, keys, firsts, aside, n_aside, seconds, bytes; };

Layout layout_of(int64_t batch, int64_t max_ctx)
{
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    Layout l;
    l.stride = (max_ctx + 63) / 64 * 64;
    l.subs = (max_ctx + kSub - 1) / kSub;
    l.segs = max_ctx > kSmall ? (max_ctx + kSeg - 1) / kSeg : 0;
    l.picked = 0;
    l.counts = up((size_t)batch * sizeof(Picked));
    l.keys = l.counts + up((size_t)batch * (size_t)l.subs * sizeof(int2));
    l.firsts = l.keys + up((size_t)batch * (size_t)l.stride * 4);
    l.parts = l.segs ? (max_ctx + kPart - 1) / kPart : 0;
    l.aside = l.firsts + up((size_t)batch * (size_t)l.segs * (kBins / 2) * 4);
    l.n_aside = l.aside + (l.segs ? up((size_t)batch * (size_t)l.stride * 4) : 0);
    l.seconds = l.n_aside + up((size_t)batch * (size_t)l.parts * 4);
    l.bytes = l.seconds + up((size_t)batch * (size_t)l.parts * (kBins / 2) * 4);
    return l;
}

} // namespace

size_t evict_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx)
{
    if (check_shape(shape) != KVS_OK || batch <= 0) return 256;
    return layout_of(batch, max_ctx).bytes;
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
    const size_t lines = (size_t)pages->batch * shape->n_kv_heads * sizeof(float);
    if (new_mass && overlap(mass, lines * mass_stride, new_mass, lines * max_keep)) return fail(KVS_EINVAL, "%s: new_mass overlaps mass", me);
    if (!workspace || workspace_bytes < evict_paged_workspace_bytes(shape, pages->batch, pg.max_ctx)) return fail(KVS_EWORKSPACE, "%s: workspace too small", me);
    const size_t pool = pool_bytes(shape, cache), ints = (size_t)pages->batch * 4;
    const Span out_mass = {new_mass, lines * max_keep, "new_mass"}, out_kept = {kept, ints * max_keep, "kept"}, out_len = {new_len, ints, "new_len"};
    const Span k = {new_table ? cache->k : nullptr, pool, "the cache's K"}, v = {new_table ? cache->v : nullptr, pool, "the cache's V"};
    const Span in_mass = {mass, lines * mass_stride, "mass"}, in_keep = {keep, ints, "keep"}, table = {pages->table, ints * pages->width, "the page table"},
               into = {new_table, ints * new_width, "new_table"}, length = {new_len == pages->ctx_len ? nullptr : pages->ctx_len, ints, "ctx_len"};
    st = check_apart(me, {out_mass, out_kept, k, v}, {in_mass, in_keep, table, into, {pages->ctx_len, ints, "ctx_len"}});
    if (st == KVS_OK) st = check_apart(me, {out_len}, {in_mass, in_keep, table, into, length, out_mass, out_kept, k, v});
    if (st == KVS_OK) st = check_apart(me, {out_kept, out_mass}, {k, v});
    if (st == KVS_OK) st = check_apart(me, {out_kept}, {out_mass});
    if (st != KVS_OK) return st;
    hipStream_t hs = (hipStream_t)stream;
    if (pg.max_ctx == 0) max_keep = 0;
    const Layout l = layout_of(pg.batch, pg.max_ctx);
    char *ws = (char *)workspace;
    Picked *picked = (Picked *)(ws + l.picked);
    int2 *counts = (int2 *)(ws + l.counts);
    uint32_t *keys = (uint32_t *)(ws + l.keys), *firsts = (uint32_t *)(ws + l.firsts);
    const dim3 threads(kThreads), requests((unsigned)pg.batch);
    if (!l.segs) {
#define KVS_SMALL(KPT)                                                                                                                                          \
    hipLaunchKernelGGL(evict_small_kernel<KPT>, requests, dim3(kSelThreads), 0, hs, pg, shape->n_kv_heads, keep, (int)max_keep, n_first, n_recent, mass, mass_stride, \
                       keys, l.stride, picked, counts, (int)l.subs, new_len)
        if (pg.max_ctx <= 4 * kSelThreads) KVS_SMALL(4);
        else if (pg.max_ctx <= 8 * kSelThreads) KVS_SMALL(8);
        else KVS_SMALL(16);
#undef KVS_SMALL
    } else {
        uint32_t *aside = (uint32_t *)(ws + l.aside), *seconds = (uint32_t *)(ws + l.seconds);
        int32_t *n_aside = (int32_t *)(ws + l.n_aside);
        hipLaunchKernelGGL(evict_keys_kernel, dim3((unsigned)l.segs, (unsigned)pg.batch), dim3(kSelThreads), 0, hs, pg, shape->n_kv_heads, keep, (int)max_keep, n_first, n_recent, mass, mass_stride,
                           keys, l.stride, firsts);
        if ((st = check_launch(me)) != KVS_OK) return st;
        hipLaunchKernelGGL(evict_scan_kernel, dim3((unsigned)l.parts, (unsigned)pg.batch), dim3(kSelThreads), 0, hs, pg, keep, (int)max_keep, keys, l.stride, firsts, (int)l.segs, aside,
                           n_aside, seconds, picked);
        if ((st = check_launch(me)) != KVS_OK) return st;
        hipLaunchKernelGGL(evict_pick_kernel, requests, dim3(kSelThreads), 0, hs, pg, keep, (int)max_keep, l.stride, aside, n_aside, seconds, (int)l.parts, picked,
                           new_len);
        if ((st = check_launch(me)) != KVS_OK) return st;
        hipLaunchKernelGGL(evict_count_kernel, dim3((unsigned)((l.subs + kWaves - 1) / kWaves), (unsigned)pg.batch), threads, 0, hs, keys, l.stride, picked, counts, (int)l.subs);
    }
    if ((st = check_launch(me)) != KVS_OK) return st;
    if (max_keep == 0 || (!new_table && !new_mass && !kept)) return KVS_OK;
    const int ppr = (int)(shape->n_kv_heads * shape->head_dim * (int64_t)elem_bytes(shape->dtype) / 16);
    const int ppl = (ppr + kWave - 1) / kWave;
    // Short contexts do not fill the chip with a workgroup for every kSub rows: several rank the same rows then, and copy a part each.  Twice as
    // many as are there at once let one rank while another copies (131072 rows: 1024 workgroups 78.0 us in all, 2048 74.1, 4096 73.8).
    int64_t parts = 4096 / (l.subs * pg.batch);
    parts = parts < 1 || !new_table ? 1 : parts > 8 ? 8 : parts;
#define KVS_MOVE(P, R)                                                                                                                            \
    hipLaunchKernelGGL((evict_move_kernel<P, R>), dim3((unsigned)l.subs, (unsigned)pg.batch, (unsigned)parts), threads, 0, hs, pg, shape->n_kv_heads, ppr, keys, l.stride, picked, counts, (int)l.subs, \
                       new_table, new_width, (uint4 *)cache->k, (uint4 *)cache->v, mass, mass_stride, kept, new_mass, (int)max_keep)
    if (ppl <= 1) KVS_MOVE(1, 8);
    else if (ppl <= 2) KVS_MOVE(2, 4);
    else if (ppl <= 4) KVS_MOVE(4, 2);
    else if (ppl <= 8) KVS_MOVE(8, 1);
    else if (ppl <= 16) KVS_MOVE(16, 1);
    else KVS_MOVE(32, 1);
#undef KVS_MOVE
    return check_launch(me);
}
