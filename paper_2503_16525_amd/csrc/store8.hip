// kvs_store_kv8: rows of K and V into a cache held in 8 bits with a scale for each block of tokens and KV head.
//
// A block's scale comes from the largest magnitude among the rows that it takes, so its rows are needed twice: once for
// that maximum and once to be divided by it.  They stay in registers in between, so memory sees them once: 2 or 4 bytes
// an element in, 1 byte out, plus the kept rows' codes where a block's scale grows.
//
// One workgroup of four waves serves one block's worth of the list (a run: the entries of one block) and walks over the
// block's units, a unit being one KV head of K or of V; `split` workgroups share a run's units.  A wave holds up to 32
// of a unit's rows, so a unit takes 1, 2 or 4 waves (`waves`) and 4 / waves units are in work at once; units of several
// waves meet in LDS for their maximum.  Which entry of the list a row of the block takes is settled first, in LDS: the
// highest entry that names it, whatever order the entries come in.
#include "cache8.h"

#include <math.h>

namespace kvs {
namespace {

constexpr int kThreads = 256;
constexpr int kWaveRows = 32;
constexpr int kMaxBlock = 128;

struct StoreArgs {
    const void *k_new, *v_new;
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    uint8_t *reused;
    float *dev_v;
    const int32_t *sel_pos;
    int64_t row0, n_sel, n_rows;
    int32_t n_kv_heads, block, waves;
};

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    return v;
}

template <int DTYPE, int CODE, int D>
__global__ __launch_bounds__(kThreads) void store_kernel(const StoreArgs a)
{
    constexpr int E = DTYPE == KVS_BF16 ? 8 : 4;           // elements of a 16-byte piece
    constexpr int PPR = D / E;                             // pieces of a row
    constexpr int RPI = kWave / PPR;                       // rows a wave loads at once
    constexpr int N = kWaveRows / RPI;                     // pieces a lane holds
    __shared__ int src[kMaxBlock];                         // entry that row r of the block takes, -1: the row is kept
    __shared__ uint32_t most_s[2][4];
    __shared__ float old_s[2][4];
    __shared__ int cut_s;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = a.block;

    // ---- the run, and what each of the block's rows takes --------------------------------------------------
    int64_t blk;
    if (a.sel_pos) {
        const int64_t s0 = blockIdx.x;
        const int64_t p = a.sel_pos[s0];
        if (p < 0 || p >= a.n_rows) return;
        blk = p / block;
        if (s0 > 0) {
            const int64_t before = a.sel_pos[s0 - 1];
            if (before >= 0 && before < a.n_rows && before / block == blk) return;     // not where a run begins
        }
        if (tid < kMaxBlock) src[tid] = -1;
        __syncthreads();
        for (int64_t s = s0;; s += kThreads) {
            const int64_t e = s + tid;
            const int64_t pe = e < a.n_sel ? (int64_t)a.sel_pos[e] : -1;
            const bool mine = pe >= 0 && pe < a.n_rows && pe / block == blk;
            // this round's first entry outside the run ends it
            if (tid == 0) cut_s = kThreads;
            __syncthreads();
            if (!mine) atomicMin(&cut_s, tid);
            __syncthreads();
            const int cut = cut_s;
            if (tid < cut) atomicMax(&src[(int)(pe - blk * block)], (int)e);
            __syncthreads();
            if (cut < kThreads) break;
        }
    } else {
        blk = a.row0 / block + blockIdx.x;
        if (tid < kMaxBlock) {
            const int64_t e = blk * block + tid - a.row0;
            src[tid] = tid < block && e >= 0 && e < a.n_sel ? (int)e : -1;
        }
        __syncthreads();
    }
    const int rows_here = (int)min((int64_t)block, a.n_rows - blk * block);
    const bool keeps = __syncthreads_or(tid < rows_here && src[tid < kMaxBlock ? tid : 0] < 0) != 0;

    if (blockIdx.y == 0) {
        for (int e = tid; e < rows_here * (a.n_kv_heads + 1); e += kThreads) {
            const int r = e % rows_here, g = e / rows_here;
            if (src[r] < 0) continue;
            if (g < a.n_kv_heads) { if (a.dev_v) a.dev_v[(int64_t)g * a.n_rows + blk * block + r] = 0.f; }
            else if (a.reused) a.reused[blk * block + r] = 0;
        }
    }

    // ---- unit by unit ----------------------------------------------------------------------------------------
    const int per_round = 4 / a.waves, mine = wave / a.waves, part = wave % a.waves;
    const int units = 2 * a.n_kv_heads;
    const int first_row = part * kWaveRows;
    int parity = 0;
    for (int u0 = (int)blockIdx.y * per_round; u0 < units; u0 += (int)gridDim.y * per_round, parity ^= 1) {
        const int u = u0 + mine;
        const bool live = u < units;
        const bool is_v = u >= a.n_kv_heads;
        const int g = is_v ? u - a.n_kv_heads : u;
        const uint4 *from = reinterpret_cast<const uint4 *>(is_v ? a.v_new : a.k_new);
        uint4 w[N];
        uint32_t bits = 0;
        const int piece = lane % PPR, sub = lane / PPR;
        if (live) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = first_row + i * RPI + sub;
                const int e = r < rows_here ? src[r] : -1;
                w[i] = make_uint4(0u, 0u, 0u, 0u);
                if (e >= 0) w[i] = stream_load16(from + ((int64_t)e * a.n_kv_heads + g) * PPR + piece);
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
        float *const scale_at = (is_v ? a.v_scale : a.k_scale) + blk * a.n_kv_heads + g;
        float old = live && lane == 0 && part == 0 ? *scale_at : 0.f;
        if (a.waves > 1) {
            // the old scale is read by the wave that will write the new one, and has arrived before the barrier; two sets in
            // turn: a wave writes to one again only behind the barrier of the round in between
            if (lane == 0) { most_s[parity][wave] = bits; old_s[parity][wave] = old; }
            __syncthreads();
            for (int i = 0; i < a.waves; ++i) bits = max(bits, most_s[parity][mine * a.waves + i]);
            old = old_s[parity][mine * a.waves];
        } else {
            old = __shfl(old, 0);
        }
        if (!live) continue;

        const float most = __uint_as_float(bits);
        const bool odd = bits >= 0x7f800000u || (keeps && old != old);
        const float need = most > 0.f ? fmaxf(most / top_code<CODE>(), kLeastScale) : 0.f;
        float scale = keeps ? fmaxf(old, need) : need;
        if (odd) scale = __uint_as_float(0x7fc00000u);
        const float inv = scale > 0.f ? 1.f / scale : 0.f;   // a NaN scale: codes of 0
        uint8_t *to = (is_v ? a.v : a.k) + (blk * block * a.n_kv_heads + g) * D;
        const int64_t row_bytes = (int64_t)a.n_kv_heads * D;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = first_row + i * RPI + sub;
            if (r >= rows_here || src[r] < 0) continue;
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
            for (int e = lane; e < kWaveRows * CP; e += kWave) {
                const int r = first_row + e / CP;
                if (r >= rows_here || src[r] >= 0) continue;
                uint4 *at = reinterpret_cast<uint4 *>(to + r * row_bytes) + e % CP;
                const uint4 c = *at;
                const uint32_t cc[4] = {c.x, c.y, c.z, c.w};
                uint32_t out[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float x[4];
                    widen_codes<CODE>(CODE == KVS_E4M3 ? numbers_only(cc[j]) : cc[j], x);
                    out[j] = nearest_codes<CODE>(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
                }
                *at = make_uint4(out[0], out[1], out[2], out[3]);
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
    const int block = cache->block;
    StoreArgs a = {k_new, v_new, (uint8_t *)cache->k, (uint8_t *)cache->v, cache->k_scale, cache->v_scale, reused, dev_v, sel_pos,
                   row0, n_sel, cache->n_rows, shape->n_kv_heads, block, block <= kWaveRows ? 1 : block / kWaveRows};
    const int64_t runs = sel_pos ? n_sel : (row0 + n_sel - 1) / block - row0 / block + 1;
    const int per_round = 4 / a.waves, rounds = (2 * a.n_kv_heads + per_round - 1) / per_round;
    // workgroups to a run: 1024 in all keep the compute units busy, and a run has no more rounds to share
    int64_t split = (1024 + runs - 1) / runs;
    if (split > rounds) split = rounds;
    hipStream_t hs = (hipStream_t)stream;
#define KVS_STORE(DT, C, DD) hipLaunchKernelGGL((store_kernel<DT, C, DD>), dim3((unsigned)runs, (unsigned)split), dim3(kThreads), 0, hs, a)
#define KVS_STORE_D(DT, C) do { if (shape->head_dim == 128) KVS_STORE(DT, C, 128); else KVS_STORE(DT, C, 64); } while (0)
    if (shape->dtype == KVS_BF16) { if (cache->code == KVS_E4M3) KVS_STORE_D(KVS_BF16, KVS_E4M3); else KVS_STORE_D(KVS_BF16, KVS_INT8); }
    else { if (cache->code == KVS_E4M3) KVS_STORE_D(KVS_F32, KVS_E4M3); else KVS_STORE_D(KVS_F32, KVS_INT8); }
#undef KVS_STORE_D
#undef KVS_STORE
    return check_launch("kvs_store_kv8");
}
