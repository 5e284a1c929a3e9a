// kvs_store_kv8: rows of K and V into a cache held in 8 bits with a scale for each block of tokens and KV head.
//
// A block's scale comes from the largest magnitude among the rows that it takes, so its rows are needed twice: once for
// that maximum and once to be divided by it.  They stay in registers in between, so memory sees them once: 2 or 4 bytes
// an element in, 1 byte out, plus the kept rows' codes where a block's scale grows.
//
// The work is a list of tasks: a run (the entries of one block) and a unit (one KV head of K or of V).  A wave holds up to
// 32 rows of a task, so a task takes a team of 1, 2 or 4 waves (`waves`); larger teams meet in LDS for their maximum.  Without a
// list a workgroup has one block and its share of the units; with one it has a chunk of the list, whose runs it finds from
// one load of the positions, and one unit or more.  Which entry a row takes is settled in LDS: the highest that names it,
// whatever order the entries of a block come in.  (A workgroup for each entry, of which those that do not begin a run end
// at once, took 35.6 us for 4424 of 32768 rows of 8 heads; this takes STORE_US.)
#include "cache8.h"

#include <math.h>

namespace kvs {
namespace {

constexpr int kThreads = 256;
constexpr int kWaveRows = 32;
constexpr int64_t kManyWgs = 4096;
constexpr int kMaxChunk = 32;          // entries of a chunk: runs that go on behind it are followed

struct StoreArgs {
    const void *k_new, *v_new;
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    uint8_t *reused;
    float *dev_v;
    const int32_t *sel_pos;
    int64_t row0, n_sel, n_rows;
    int32_t n_kv_heads, block_log2, waves, units_per_wg, chunk;
};

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    return v;
}

template <int DTYPE, int CODE, int D, bool LIST>
__global__ __launch_bounds__(kThreads) void store_kernel(const StoreArgs a)
{
    constexpr int E = DTYPE == KVS_BF16 ? 8 : 4;           // elements of a 16-byte piece
    constexpr int PPR = D / E;                             // pieces of a row
    constexpr int RPI = kWave / PPR;                       // rows a wave loads at once
    constexpr int N = kWaveRows / RPI;                     // pieces a lane holds
    __shared__ int src_s[4][kWaveRows];                    // entry that a row of the wave's part takes, -1: the row is kept
    __shared__ uint32_t most_s[2][4];
    __shared__ float old_s[2][4];
    __shared__ int keeps_s[2][4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = 1 << a.block_log2, hk = a.n_kv_heads, units = 2 * hk;
    const int n_teams = 4 / a.waves, team = wave / a.waves, part = wave % a.waves, first_row = part * kWaveRows;

    // ---- the runs ---------------------------------------------------------------------------------------------------
    // lane i holds entry chunk0 + i: its block (-1: outside the cache), and whether a run begins there
    const int64_t chunk0 = LIST ? (int64_t)blockIdx.x * a.chunk : 0;
    int64_t my_blk = -1;
    int my_pos = -1;
    uint64_t begins = 1;
    int n_runs = 1;
    if constexpr (LIST) {
        const int64_t e = chunk0 + lane;
        my_pos = e < a.n_sel ? a.sel_pos[e] : -1;
        const int before = lane == 0 && chunk0 > 0 ? a.sel_pos[chunk0 - 1] : -1;
        auto blk_of = [&](int p) -> int64_t { return p >= 0 && p < a.n_rows ? (int64_t)(p >> a.block_log2) : -1; };
        my_blk = blk_of(my_pos);
        int64_t left = __shfl_up((int)my_blk, 1);
        if (lane == 0) left = blk_of(before);
        begins = __ballot(my_blk != left || my_blk < 0);
        const uint64_t mine = __ballot(my_blk >= 0 && lane < a.chunk && my_blk != left);
        n_runs = __popcll(mine);
        if (blockIdx.y == 0 && wave == 0 && my_blk >= 0 && lane < a.chunk) {
            if (a.reused) a.reused[my_pos] = 0;
            if (a.dev_v) for (int g = 0; g < hk; ++g) a.dev_v[(int64_t)g * a.n_rows + my_pos] = 0.f;
        }
        if (n_runs == 0) return;                            // the same in all waves
    } else if (blockIdx.y == 0) {
        const int64_t first = max((a.row0 >> a.block_log2) + blockIdx.x, (int64_t)0) << a.block_log2;
        for (int e = tid; e < block * (hk + 1); e += kThreads) {
            const int64_t r = first + (e & (block - 1));
            const int g = e >> a.block_log2;
            if (r < a.row0 || r >= a.row0 + a.n_sel) continue;
            if (g < hk) { if (a.dev_v) a.dev_v[(int64_t)g * a.n_rows + r] = 0.f; }
            else if (a.reused) a.reused[r] = 0;
        }
    }

    const int u_lo = (int)blockIdx.y * a.units_per_wg, n_units = min(a.units_per_wg, units - u_lo);
    const int n_tasks = n_runs * n_units;
    int *const src = src_s[wave];
    int run_of_src = -1, parity = 0;
    bool keeps_part = false;
    int64_t blk = LIST ? 0 : (a.row0 >> a.block_log2) + blockIdx.x;
    int rows_here = 0;
    for (int k0 = 0; k0 < n_tasks; k0 += n_teams, parity ^= 1) {
        const int task = k0 + team;
        const bool live = task < n_tasks;
        const int run = live ? task / n_units : 0, u = u_lo + (live ? task - run * n_units : 0);
        if (live && run != run_of_src) {
            run_of_src = run;
            if (lane < kWaveRows) src[lane] = -1;
            asm volatile("" ::: "memory");                  // (LDS works a wave's accesses off in order)
            if constexpr (LIST) {
                // the run-th place where a run of this chunk begins, and where the next one does
                uint64_t left = __ballot(my_blk >= 0 && lane < a.chunk && ((begins >> lane) & 1));
                for (int i = 0; i < run; ++i) left &= left - 1;
                const int at = __builtin_ctzll(left);
                const uint64_t after = at == 63 ? 0 : begins >> (at + 1);
                const int end = after ? at + 1 + __builtin_ctzll(after) : 64;
                blk = __builtin_amdgcn_readlane((int)my_blk, at);
                const int base = (int)(blk << a.block_log2) + first_row;       // rows are int32 in a list
                if (lane >= at && lane < end && (uint32_t)(my_pos - base) < (uint32_t)kWaveRows) atomicMax(&src[my_pos - base], (int)(chunk0 + lane));
                if (end == 64) {
                    for (int64_t s = chunk0 + 64;; s += 64) {
                        const int64_t e = s + lane;
                        const int p = e < a.n_sel ? a.sel_pos[e] : -1;
                        const bool in = p >= 0 && p < a.n_rows && (p >> a.block_log2) == (int)blk;
                        const uint64_t out = __ballot(!in);
                        const int cut = out ? __builtin_ctzll(out) : 64;
                        if (lane < cut && (uint32_t)(p - base) < (uint32_t)kWaveRows) atomicMax(&src[p - base], (int)e);
                        if (cut < 64) break;
                    }
                }
            } else if (lane < kWaveRows) {
                const int64_t e = (blk << a.block_log2) + first_row + lane - a.row0;
                src[lane] = first_row + lane < block && e >= 0 && e < a.n_sel ? (int)e : -1;
            }
            asm volatile("" ::: "memory");
            rows_here = (int)min((int64_t)block, a.n_rows - (blk << a.block_log2)) - first_row;     // from the wave's first row on
            keeps_part = __ballot(lane < kWaveRows && lane < rows_here && src[lane & (kWaveRows - 1)] < 0) != 0;
        }

        const bool is_v = u >= hk;
        const int g = is_v ? u - hk : u;
        float *const scale_at = (is_v ? a.v_scale : a.k_scale) + blk * hk + g;
        float old = 0.f;
        if (live && part == 0) old = *scale_at;
        const uint4 *from = reinterpret_cast<const uint4 *>(is_v ? a.v_new : a.k_new);
        uint4 w[N];
        uint32_t bits = 0;
        const int piece = lane % PPR, sub = lane / PPR;
        if (live) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = i * RPI + sub, e = src[r];
                w[i] = make_uint4(0u, 0u, 0u, 0u);
                if (e >= 0) w[i] = stream_load16(from + ((int64_t)e * hk + g) * PPR + piece);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t ww[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (DTYPE == KVS_BF16) bits = max(bits, max((ww[j] << 16) & 0x7fffffffu, ww[j] & 0x7fff0000u));
                    else bits = max(bits, ww[j] & 0x7fffffffu);
                }
            }
        }
        bits = wave_max_bits(bits);                         // magnitudes order as whole numbers, NaN above infinity above the rest
        bool keeps = keeps_part;
        if (a.waves > 1) {
            // the old scale is read by the wave that will write the new one, and has arrived before the barrier; two sets in
            // turn: a wave writes to one again only behind the barrier of the round in between
            if (lane == 0) { most_s[parity][wave] = bits; old_s[parity][wave] = old; keeps_s[parity][wave] = keeps_part; }
            __syncthreads();
            for (int i = 0; i < a.waves; ++i) {
                bits = max(bits, most_s[parity][team * a.waves + i]);
                keeps |= keeps_s[parity][team * a.waves + i] != 0;
            }
            old = old_s[parity][team * a.waves];
        }
        if (!live) continue;

        const float most = __uint_as_float(bits);
        const bool odd = bits >= 0x7f800000u || (keeps && old != old);
        const float need = most > 0.f ? fmaxf(most * (1.f / top_code<CODE>()), kLeastScale) : 0.f;
        float scale = keeps ? fmaxf(old, need) : need;
        if (odd) scale = __uint_as_float(0x7fc00000u);
        const float inv = scale > 0.f ? 1.f / scale : 0.f;   // a NaN scale: codes of 0
        const int64_t row_bytes = (int64_t)hk * D;
        uint8_t *to = (is_v ? a.v : a.k) + (((blk << a.block_log2) + first_row) * hk + g) * D;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = i * RPI + sub;
            if (src[r] < 0) continue;
            uint8_t *dst = to + r * row_bytes + piece * E;
            if constexpr (DTYPE == KVS_BF16) {
                uint2 c;
                c.x = nearest_codes<CODE>(bf16_lo(w[i].x) * inv, bf16_hi(w[i].x) * inv, bf16_lo(w[i].y) * inv, bf16_hi(w[i].y) * inv);
                c.y = nearest_codes<CODE>(bf16_lo(w[i].z) * inv, bf16_hi(w[i].z) * inv, bf16_lo(w[i].w) * inv, bf16_hi(w[i].w) * inv);
                if (odd) c = make_uint2(0u, 0u);
                *reinterpret_cast<uint2 *>(dst) = c;
            } else {
                uint32_t c = nearest_codes<CODE>(__uint_as_float(w[i].x) * inv, __uint_as_float(w[i].y) * inv, __uint_as_float(w[i].z) * inv, __uint_as_float(w[i].w) * inv);
                if (odd) c = 0u;
                *reinterpret_cast<uint32_t *>(dst) = c;
            }
        }
        // kept rows stand for what they stood for, in steps of the new scale
        if (keeps && !odd && scale > 0.f && scale != old) {
            const float ratio = old / scale;
            constexpr int CP = D / 16;                       // 16-byte pieces of a row of codes
            uint4 held[kWaveRows * CP / kWave];
#pragma unroll
            for (int i = 0; i < kWaveRows * CP / kWave; ++i) {
                const int e = lane + i * kWave, r = e / CP;
                held[i] = make_uint4(0u, 0u, 0u, 0u);
                if (r < rows_here && src[r] < 0) held[i] = reinterpret_cast<const uint4 *>(to + r * row_bytes)[e % CP];
            }
#pragma unroll
            for (int i = 0; i < kWaveRows * CP / kWave; ++i) {
                const int e = lane + i * kWave, r = e / CP;
                if (r >= rows_here || src[r] >= 0) continue;
                const uint32_t cc[4] = {held[i].x, held[i].y, held[i].z, held[i].w};
                uint32_t out[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float x[4];
                    widen_codes<CODE>(CODE == KVS_E4M3 ? numbers_only(cc[j]) : cc[j], x);
                    out[j] = nearest_codes<CODE>(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
                }
                reinterpret_cast<uint4 *>(to + r * row_bytes)[e % CP] = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
        if (lane == 0 && part == 0) *scale_at = scale;
    }
}

} // namespace
} // namespace kvs

kvs_status kvs::check_cache8(const char *me, const kvs_shape *shape, const kvs_cache8 *c)
{
    if (!c) return fail(KVS_EINVAL, "%s: cache is NULL", me);
    if (c->code != KVS_E4M3 && c->code != KVS_INT8) return fail(KVS_EINVAL, "%s: unknown code %d", me, c->code);
    if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128)
        return fail(KVS_EINVAL, "%s: blocks of %d tokens (16, 32, 64 and 128 are built)", me, c->block);
    if (c->n_rows < 0) return fail(KVS_EINVAL, "%s: n_rows < 0", me);
    if (shape->n_kv_heads > 64) return fail(KVS_EUNSUPPORTED, "%s: more than 64 kv heads", me);
    if (c->n_rows > ((int64_t)1 << 40) / (shape->n_kv_heads * shape->head_dim)) return fail(KVS_EUNSUPPORTED, "%s: a cache of %lld rows", me, (long long)c->n_rows);
    if (c->n_rows == 0) return KVS_OK;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(KVS_EINVAL, "%s: NULL pointer in the cache", me);
    if (!aligned16(c->k) || !aligned16(c->v)) return fail(KVS_EINVAL, "%s: the cache's codes must be 16-byte aligned", me);
    if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 3u) return fail(KVS_EINVAL, "%s: misaligned scales", me);
    return KVS_OK;
}

extern "C" kvs_status kvs_store_kv8(const kvs_shape *shape, const kvs_cache8 *cache, const void *k_new, const void *v_new,
                                    const int32_t *sel_pos, int64_t row0, int64_t n_sel,
                                    uint8_t *reused, float *dev_v, void *stream)
{
    using namespace kvs;
    kvs_status st = check_shape(shape);
    if (st != KVS_OK || (st = check_cache8("kvs_store_kv8", shape, cache)) != KVS_OK) return st;
    if (n_sel < 0 || n_sel > 0x7fffffff) return fail(KVS_EINVAL, "kvs_store_kv8: n_sel %lld", (long long)n_sel);
    if (!sel_pos && (row0 < 0 || row0 > cache->n_rows - n_sel))
        return fail(KVS_EINVAL, "kvs_store_kv8: rows %lld .. +%lld of a cache of %lld", (long long)row0, (long long)n_sel, (long long)cache->n_rows);
    if (n_sel == 0 || cache->n_rows == 0) return KVS_OK;
    if (!k_new || !v_new) return fail(KVS_EINVAL, "kvs_store_kv8: NULL pointer");
    if (!aligned16(k_new) || !aligned16(v_new)) return fail(KVS_EINVAL, "kvs_store_kv8: K/V pointers must be 16-byte aligned");
    const int block = cache->block, waves = block <= kWaveRows ? 1 : block / kWaveRows, teams = 4 / waves, units = 2 * shape->n_kv_heads;
    StoreArgs a = {k_new, v_new, (uint8_t *)cache->k, (uint8_t *)cache->v, cache->k_scale, cache->v_scale, reused, dev_v, sel_pos,
                   row0, n_sel, cache->n_rows, shape->n_kv_heads, __builtin_ctz((unsigned)block), waves, 1, 1};
    int64_t wgs;
    if (sel_pos) {
        // a unit a workgroup; chunks that give a team one run, longer ones once there are more workgroups than the chip holds
        int64_t chunk = teams;
        while (chunk < kMaxChunk && (n_sel / chunk) * units > kManyWgs) chunk *= 2;
        a.chunk = (int)chunk;
        wgs = (n_sel + chunk - 1) / chunk;
    } else {
        // 1024 workgroups keep the compute units busy, and a block has no more rounds to share
        wgs = (row0 + n_sel - 1) / block - row0 / block + 1;
        const int64_t rounds = (units + teams - 1) / teams;
        int64_t split = (1024 + wgs - 1) / wgs;
        if (split > rounds) split = rounds;
        a.units_per_wg = (int)((rounds + split - 1) / split) * teams;
    }
    const dim3 grid((unsigned)wgs, (unsigned)((units + a.units_per_wg - 1) / a.units_per_wg));
    hipStream_t hs = (hipStream_t)stream;
#define KVS_STORE(DT, C, DD)                                                                                          \
    do {                                                                                                              \
        if (sel_pos) hipLaunchKernelGGL((store_kernel<DT, C, DD, true>), grid, dim3(kThreads), 0, hs, a);              \
        else hipLaunchKernelGGL((store_kernel<DT, C, DD, false>), grid, dim3(kThreads), 0, hs, a);                     \
    } while (0)
#define KVS_STORE_D(DT, C) do { if (shape->head_dim == 128) KVS_STORE(DT, C, 128); else KVS_STORE(DT, C, 64); } while (0)
    if (shape->dtype == KVS_BF16) { if (cache->code == KVS_E4M3) KVS_STORE_D(KVS_BF16, KVS_E4M3); else KVS_STORE_D(KVS_BF16, KVS_INT8); }
    else { if (cache->code == KVS_E4M3) KVS_STORE_D(KVS_F32, KVS_E4M3); else KVS_STORE_D(KVS_F32, KVS_INT8); }
#undef KVS_STORE_D
#undef KVS_STORE
    return check_launch("kvs_store_kv8");
}
