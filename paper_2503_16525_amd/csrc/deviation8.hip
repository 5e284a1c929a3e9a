// kvs_deviation_kv8: per-token, per-KV-head L1 deviation of freshly computed K/V from what a cache in 8 bits holds, and the
// score of Alg. 1 step 3 from it.
//
// A stream over two tensors: fresh rows of 2 or 4 bytes an element, codes of 1, a scale for each block and head.  Cells
// (token, head) are contiguous on both sides, so a lane takes a 16-byte piece of the fresh cell and the 8 or 4 codes
// that belong to it; kCells cells are in flight a lane.  The lanes of a cell meet by DPP in a fixed order, the tile's sums
// pass through LDS so that dev_* leave along the tokens, and the score is summed head by head.  (V of 32768 tokens of 8 heads,
// cold: 18.5 us, 5.5 TB/s; 131072 tokens of 4 heads 34.)
#include "cache8.h"

#include <math.h>

namespace kvs {
namespace {

constexpr int kThreads = 256;
// Tokens of a workgroup's tile: 8, from 8 heads on 4, which are 32 cells and two a lane.  V in bf16, tiles of 4 and 8 (and 16): 131072 tokens of 1
// head 28.4 and 16.9 us (11.2), 2 heads 31.3 and 19.9 (18.0), 3 heads 33.8 and 27.2 (25.6), 4 heads 37.0 and 31.5 (32.6); 65536 of 5
// heads 25.2 and 22.7, 6 heads 27.3 and 25.6, 7 heads 29.4 and 30.4, 8 heads 31.8 and 32.8; 32768 of 12 heads 26.1 and 25.8, 16
// heads 33.3 and 34.1, 32 heads 62.7 and 62.9; 12000 of 8 heads 9.2 and 9.6 (9.9, with 32 14.6); 8192 of 16 heads 11.7 and 11.4
// (15.2).  Above 8 heads either would do, and larger tiles leave units idle in short launches.
constexpr int kTok = 8, kTokMany = 4, kManyHeads = 8;

struct DevArgs {
    const void *k_fresh, *v_fresh;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    const uint8_t *reused;
    const float *alpha;
    float *dev_k, *dev_v, *score;
    int64_t row0, n_tokens;
    int32_t n_kv_heads, block_log2, mode_kv;
};

template <int LPH>
__device__ __forceinline__ float cell_sum(float v)
{
    if (LPH == 16) return row16_sum(v);
    if (LPH == 32) { v = row16_sum(v); return v + __shfl_xor(v, 16); }
    v += __shfl_xor(v, 4);
    v += __shfl_xor(v, 2);
    return v + __shfl_xor(v, 1);
}

// sum of |fresh - code * scale| over a 16-byte piece of fresh values
template <int DTYPE, int CODE>
__device__ __forceinline__ float l1_piece(const uint4 f, const uint32_t c0, const uint32_t c1, float scale)
{
    float x[4], y[4];
    widen_codes<CODE>(c0, x);
    if constexpr (DTYPE == KVS_BF16) {
        widen_codes<CODE>(c1, y);
        const float s0 = fabsf(fmaf(-x[0], scale, bf16_lo(f.x))) + fabsf(fmaf(-x[1], scale, bf16_hi(f.x)));
        const float s1 = fabsf(fmaf(-x[2], scale, bf16_lo(f.y))) + fabsf(fmaf(-x[3], scale, bf16_hi(f.y)));
        const float s2 = fabsf(fmaf(-y[0], scale, bf16_lo(f.z))) + fabsf(fmaf(-y[1], scale, bf16_hi(f.z)));
        const float s3 = fabsf(fmaf(-y[2], scale, bf16_lo(f.w))) + fabsf(fmaf(-y[3], scale, bf16_hi(f.w)));
        return (s0 + s1) + (s2 + s3);
    } else {
        const float s0 = fabsf(fmaf(-x[0], scale, __uint_as_float(f.x))) + fabsf(fmaf(-x[1], scale, __uint_as_float(f.y)));
        const float s1 = fabsf(fmaf(-x[2], scale, __uint_as_float(f.z))) + fabsf(fmaf(-x[3], scale, __uint_as_float(f.w)));
        return s0 + s1;
    }
}

template <int DTYPE, int CODE, int D, bool HAS_K, int TOK>
__global__ __launch_bounds__(kThreads) void deviation8_kernel(const DevArgs a)
{
    constexpr int E = DTYPE == KVS_BF16 ? 8 : 4;
    constexpr int LPH = D / E;                             // lanes of a cell
    constexpr int CPB = kThreads / LPH;                    // cells of a step
    constexpr int kCells = HAS_K ? 2 : 4;
    extern __shared__ float sums[];                        // dv[n_kv_heads][TOK], then dk
    const int hk = a.n_kv_heads;
    float *dv_s = sums, *dk_s = sums + hk * TOK;
    const int tid = threadIdx.x, sub = tid % LPH, cell_in_step = tid / LPH;
    const int64_t tok0 = (int64_t)blockIdx.x * TOK;
    const int toks = (int)min((int64_t)TOK, a.n_tokens - tok0);
    const int cells = toks * hk;
    const uint4 *vf = (const uint4 *)a.v_fresh + tok0 * hk * LPH, *kf = (const uint4 *)a.k_fresh + tok0 * hk * LPH;
    const uint8_t *vc = a.v + (a.row0 + tok0) * hk * D, *kc = a.k + (a.row0 + tok0) * hk * D;
    const uint8_t is_reused = a.reused && tid < toks ? a.reused[tok0 + tid] : (uint8_t)1;

    auto codes = [](const uint8_t *p) -> uint2 {
        if constexpr (E == 8) return *reinterpret_cast<const uint2 *>(p);
        else return make_uint2(*reinterpret_cast<const uint32_t *>(p), 0u);
    };
    for (int base = 0; base < cells; base += CPB * kCells) {
        uint4 v[kCells], k[kCells];
        uint2 v8[kCells], k8[kCells];
        float vs[kCells], ks[kCells];
#pragma unroll
        for (int i = 0; i < kCells; ++i) {
            const int c = base + i * CPB + cell_in_step;
            if (c >= cells) continue;
            const int t = c / hk, g = c - t * hk;
            const int64_t at = ((a.row0 + tok0 + t) >> a.block_log2) * hk + g;
            v[i] = stream_load16(vf + (int64_t)c * LPH + sub);
            v8[i] = codes(vc + (int64_t)c * D + sub * E);
            vs[i] = a.v_scale[at];
            if (HAS_K) {
                k[i] = stream_load16(kf + (int64_t)c * LPH + sub);
                k8[i] = codes(kc + (int64_t)c * D + sub * E);
                ks[i] = a.k_scale[at];
            }
        }
#pragma unroll
        for (int i = 0; i < kCells; ++i) {
            const int c = base + i * CPB + cell_in_step;   // the same in all lanes of a cell
            float sv = 0.f, sk = 0.f;
            if (c < cells) {
                // a block of scale 0 stands for zeros whatever its codes
                sv = l1_piece<DTYPE, CODE>(v[i], vs[i] != 0.f ? v8[i].x : 0u, vs[i] != 0.f ? v8[i].y : 0u, vs[i]);
                if (HAS_K) sk = l1_piece<DTYPE, CODE>(k[i], ks[i] != 0.f ? k8[i].x : 0u, ks[i] != 0.f ? k8[i].y : 0u, ks[i]);
            }
            sv = cell_sum<LPH>(sv);
            if (HAS_K) sk = cell_sum<LPH>(sk);
            if (c < cells && sub == 0) {
                const int t = c / hk, g = c - t * hk;
                dv_s[g * TOK + t] = sv;
                if (HAS_K) dk_s[g * TOK + t] = sk;
            }
        }
    }
    __syncthreads();
    for (int e = tid; e < hk * TOK; e += kThreads) {
        const int g = e / TOK, t = e % TOK;
        if (t >= toks) continue;
        const int64_t o = (int64_t)g * a.n_tokens + tok0 + t;
        if (a.dev_v) a.dev_v[o] = dv_s[e];
        if (HAS_K && a.dev_k) a.dev_k[o] = dk_s[e];
    }
    if (a.score && tid < toks) {
        float s = 0.f;
        for (int g = 0; g < hk; ++g) {
            float dev = dv_s[g * TOK + tid];
            if (HAS_K && a.mode_kv) dev = dk_s[g * TOK + tid] + dev;
            s += (a.alpha ? a.alpha[(int64_t)g * a.n_tokens + tok0 + tid] : 1.f) * dev;
        }
        a.score[tok0 + tid] = is_reused != 0 ? s : -INFINITY;
    }
}

template <int DTYPE, int CODE, int D>
kvs_status launch(const DevArgs &a, bool has_k, hipStream_t hs)
{
    const bool many = a.n_kv_heads >= kManyHeads;
    const int tok = many ? kTokMany : kTok;
    const int64_t wgs = (a.n_tokens + tok - 1) / tok;
    if (wgs > kMostWgs) return fail(KVS_EUNSUPPORTED, "kvs_deviation_kv8: %lld tokens in one call", (long long)a.n_tokens);
    const size_t lds = sizeof(float) * a.n_kv_heads * tok * 2;
#define KVS_DEV8(HASK, TOK) hipLaunchKernelGGL((deviation8_kernel<DTYPE, CODE, D, HASK, TOK>), dim3((unsigned)wgs), dim3(kThreads), lds, hs, a)
    if (has_k) { if (many) KVS_DEV8(true, kTokMany); else KVS_DEV8(true, kTok); }
    else { if (many) KVS_DEV8(false, kTokMany); else KVS_DEV8(false, kTok); }
#undef KVS_DEV8
    return check_launch("kvs_deviation_kv8");
}

} // namespace
} // namespace kvs

extern "C" kvs_status kvs_deviation_kv8(const kvs_shape *shape, const kvs_cache8 *cache, int64_t row0, int64_t n_tokens,
                                        const void *k_fresh, const void *v_fresh,
                                        const uint8_t *reused, const float *alpha, int32_t mode,
                                        float *dev_k, float *dev_v, float *score, void *stream)
{
    using namespace kvs;
    kvs_status st = check_shape(shape);
    if (st != KVS_OK || (st = check_cache8("kvs_deviation_kv8", shape, cache)) != KVS_OK) return st;
    if (mode != KVS_SCORE_V && mode != KVS_SCORE_KV) return fail(KVS_EINVAL, "kvs_deviation_kv8: unknown mode %d", mode);
    if (n_tokens < 0 || row0 < 0 || row0 > cache->n_rows - n_tokens)
        return fail(KVS_EINVAL, "kvs_deviation_kv8: rows %lld .. +%lld of a cache of %lld", (long long)row0, (long long)n_tokens, (long long)cache->n_rows);
    if (n_tokens == 0) return KVS_OK;
    const bool has_k = mode == KVS_SCORE_KV || dev_k;
    if (!v_fresh) return fail(KVS_EINVAL, "kvs_deviation_kv8: v_fresh is NULL");
    if (has_k && !k_fresh) return fail(KVS_EINVAL, "kvs_deviation_kv8: k_fresh is NULL but the key deviation is asked for");
    if (!aligned16(v_fresh) || (has_k && !aligned16(k_fresh))) return fail(KVS_EINVAL, "kvs_deviation_kv8: K/V pointers must be 16-byte aligned");
    const DevArgs a = {k_fresh, v_fresh, (const uint8_t *)cache->k, (const uint8_t *)cache->v, cache->k_scale, cache->v_scale, reused, alpha, dev_k, dev_v, score,
                       row0, n_tokens, shape->n_kv_heads, __builtin_ctz((unsigned)cache->block), mode == KVS_SCORE_KV};
    hipStream_t hs = (hipStream_t)stream;
    const bool e4m3 = cache->code == KVS_E4M3, wide = shape->head_dim == 128;
    if (shape->dtype == KVS_BF16) {
        if (e4m3) return wide ? launch<KVS_BF16, KVS_E4M3, 128>(a, has_k, hs) : launch<KVS_BF16, KVS_E4M3, 64>(a, has_k, hs);
        return wide ? launch<KVS_BF16, KVS_INT8, 128>(a, has_k, hs) : launch<KVS_BF16, KVS_INT8, 64>(a, has_k, hs);
    }
    if (e4m3) return wide ? launch<KVS_F32, KVS_E4M3, 128>(a, has_k, hs) : launch<KVS_F32, KVS_E4M3, 64>(a, has_k, hs);
    return wide ? launch<KVS_F32, KVS_INT8, 128>(a, has_k, hs) : launch<KVS_F32, KVS_INT8, 64>(a, has_k, hs);
}
