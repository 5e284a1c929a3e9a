// kvs_mass_paged: the attention that every cached row receives from a call's tokens, added to what it received before.
//
// Mathematics.  mass[i] += sum over rows r (tokens times the query heads of the KV head) of exp(scale q_r . k_i - lse_r): the column sums
// of a softmax whose rows' sums are known.  S = Q K^T with the keys as columns, so that a column's entries lie in two lanes' registers and
// nothing is exchanged before the end; every sum belongs to one wave, in a fixed order.
//
// A wave keeps its keys as operands in registers for the whole call and the rows come by, 32 at a time, through LDS.
#include "paged.h"

#include <math.h>

namespace kvs {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kRows = 32;
constexpr int kMaxPieces = 16;
template <int DTYPE> constexpr int kBlocks = DTYPE == KVS_F32 ? 1 : 2;             // of 32 keys a wave
template <int DTYPE> constexpr int kWgKeys = 32 * kBlocks<DTYPE> * kWaves;

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8, v); }

template <int DTYPE, int D>
__global__ __launch_bounds__(kThreads, 2) void mass_paged_kernel(
    const Paged pg, int n_q_heads, int n_kv_heads, int key_blocks, int pieces, const char *__restrict__ k_pool, const char *__restrict__ q_new,
    const float *__restrict__ lse, float scale_log2, float decay, const float *mass, float *mass_out, int64_t mass_stride, float *__restrict__ part)
{
    constexpr bool F32 = DTYPE == KVS_F32;
    constexpr int ROW_B = D * (F32 ? 4 : 2);
    constexpr int CPR = ROW_B / 16;
    constexpr int NB = kBlocks<DTYPE>;
    constexpr int NS = CPR / 2;                              // products of a tile (fp32: four each)
    constexpr int NQ = kRows * CPR / kThreads;               // chunks of a row tile a thread moves
    __shared__ __attribute__((aligned(16))) char q_s[2][kRows * ROW_B];
    __shared__ __attribute__((aligned(16))) float lse_s[2][kRows];
    __shared__ __attribute__((aligned(16))) int pos_s[2][kRows];
    __shared__ int span_s[2][3];                             // lowest position, highest, lowest of those that see anything

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hf = lane >> 5, ln = lane & 31;
    const int g = (int)(blockIdx.x % (uint32_t)n_kv_heads);
    int rest = (int)(blockIdx.x / (uint32_t)n_kv_heads);
    const int kb = rest % key_blocks;
    rest /= key_blocks;
    const int piece = rest % pieces, b = rest / pieces;
    const int len = len_of(pg, b);
    const int wg_lo = kb * kWgKeys<DTYPE>;
    if (wg_lo >= len) return;
    const int wg_hi = min(wg_lo + kWgKeys<DTYPE>, len) - 1;
    int tok0, n_tok;
    tokens_of(pg, b, tok0, n_tok);
    const int grp = n_q_heads / n_kv_heads;
    const int rows = n_tok * grp;
    const int row_blocks = (rows + kRows - 1) / kRows, per_piece = (row_blocks + pieces - 1) / pieces;
    const int rb_lo = min(piece * per_piece, row_blocks), rb_hi = min(rb_lo + per_piece, row_blocks);

    // ---- keys ---------------------------------------------------------------------------------------------------
    u32x4_t kreg[NB][NS];
    bool there[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int key = wg_lo + (wave * NB + nb) * 32 + ln;
        const int at = granule_of(pg, b, key / kGranule);
        there[nb] = at >= 0 && key < len;
        const char *from = k_pool + (((int64_t)max(at, 0) * kGranule + key % kGranule) * n_kv_heads + g) * ROW_B;
#pragma unroll
        for (int c = 0; c < NS; ++c) kreg[nb][c] = *reinterpret_cast<const u32x4_t *>(from + (2 * c + hf) * 16);
    }

    // ---- rows ---------------------------------------------------------------------------------------------------
    auto swz = [](int r) { return CPR >= 16 ? (r & 15) : (r & 7); };
    struct Row { int t, h; };
    auto row_at = [&](int r) { return Row{r / grp, r % grp}; };
    const int dt = kRows / grp, dh = kRows % grp;
    auto advance = [&](Row &r) {
        r.t += dt;
        r.h += dh;
        if (r.h >= grp) { r.h -= grp; ++r.t; }
    };
    Row mine[NQ], info = row_at(rb_lo * kRows + ln);
#pragma unroll
    for (int j = 0; j < NQ; ++j) mine[j] = row_at(rb_lo * kRows + (tid + j * kThreads) / CPR);
    u32x4_t q_next[NQ];
    float lse_next = 0.f;
    int pos_next = -1;
    auto fetch = [&]() {
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
            q_next[j] = u32x4_t{0u, 0u, 0u, 0u};
            if (mine[j].t < n_tok)
                q_next[j] = *reinterpret_cast<const u32x4_t *>(q_new + ((int64_t)(tok0 + mine[j].t) * n_q_heads + g * grp + mine[j].h) * ROW_B + ((tid + j * kThreads) % CPR) * 16);
            advance(mine[j]);
        }
        if (wave == 0) {
            pos_next = -1;
            lse_next = 0.f;
            if (info.t < n_tok) {
                lse_next = lse[(int64_t)(tok0 + info.t) * n_q_heads + g * grp + info.h] * 1.4426950408889634f;
                pos_next = position_of(pg, tok0, n_tok, info.t, len);
                if (lse_next == -INFINITY) pos_next = -1;    // saw nothing
            }
            advance(info);
        }
    };
    const int window = pg.window, n_first = window ? pg.n_first : 0;
    float acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[nb] = 0.f;
    if (rb_lo < rb_hi) fetch();
    for (int rb = rb_lo; rb < rb_hi; ++rb) {
        const int buf = (rb - rb_lo) & 1;
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
            const int r = (tid + j * kThreads) / CPR, c = (tid + j * kThreads) % CPR;
            *reinterpret_cast<u32x4_t *>(q_s[buf] + r * ROW_B + (c ^ swz(r)) * 16) = q_next[j];
        }
        if (wave == 0) {
            int lo = pos_next, hi = pos_next, low = pos_next < 0 ? 0x7fffffff : pos_next;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                lo = min(lo, __shfl_xor(lo, o));
                hi = max(hi, __shfl_xor(hi, o));
                low = min(low, __shfl_xor(low, o));
            }
            if (hf == 0) { lse_s[buf][ln] = lse_next; pos_s[buf][ln] = pos_next; }
            if (lane == 0) { span_s[buf][0] = lo; span_s[buf][1] = hi; span_s[buf][2] = low; }
        }
        __syncthreads();
        if (rb + 1 < rb_hi) fetch();
        const int pmin = __builtin_amdgcn_readfirstlane(span_s[buf][0]), pmax = __builtin_amdgcn_readfirstlane(span_s[buf][1]), plow = __builtin_amdgcn_readfirstlane(span_s[buf][2]);
        if (pmax < wg_lo || (window && wg_hi <= plow - window && wg_lo >= n_first)) continue;
        const bool masked = wg_hi > pmin || (window && wg_lo <= pmax - window && wg_hi >= n_first);
        floatx16 s[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[nb][r] = 0.f;
#pragma unroll
        for (int c = 0; c < NS; ++c) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t *>(q_s[buf] + ln * ROW_B + ((2 * c + hf) ^ swz(ln)) * 16);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                if constexpr (F32) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) s[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[u]), __uint_as_float(kreg[nb][c][u]), s[nb], 0, 0, 0);
                } else {
                    s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w), as_bf16x8(kreg[nb][c]), s[nb], 0, 0, 0);
                }
            }
        }
        float sum[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) sum[nb] = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {                        // entry 4 q + u is row 8 q + 4 hf + u
            const float4 l4 = *reinterpret_cast<const float4 *>(&lse_s[buf][8 * q + 4 * hf]);
            const float l[4] = {l4.x, l4.y, l4.z, l4.w};
            const int4 p4 = *reinterpret_cast<const int4 *>(&pos_s[buf][8 * q + 4 * hf]);
            const int p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float e[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) e[u] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][4 * q + u], scale_log2, -l[u]));
                if (masked) {
                    const int key = wg_lo + (wave * NB + nb) * 32 + ln;
#pragma unroll
                    for (int u = 0; u < 4; ++u) e[u] = key <= p[u] && (!window || key > p[u] - window || key < n_first) ? e[u] : 0.f;
                }
                sum[nb] += (e[0] + e[1]) + (e[2] + e[3]);
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb] += sum[nb];
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float total = acc[nb] + __shfl_xor(acc[nb], 32);
        const int key = wg_lo + (wave * NB + nb) * 32 + ln;
        if (hf != 0 || key >= len) continue;
        if (!there[nb]) total = 0.f;
        if (pieces > 1) {
            part[(((int64_t)piece * pg.batch + b) * n_kv_heads + g) * pg.max_ctx + key] = total;
        } else {
            const int64_t at = ((int64_t)b * n_kv_heads + g) * mass_stride + key;
            mass_out[at] = mass ? __builtin_fmaf(decay, mass[at], total) : total;
        }
    }
}

__global__ __launch_bounds__(kThreads) void mass_join_kernel(const Paged pg, int n_kv_heads, int pieces, const float *__restrict__ part, float decay, const float *mass,
                                                             float *mass_out, int64_t mass_stride)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int row = blockIdx.y;                              // request and KV head
    if (i >= len_of(pg, row / n_kv_heads)) return;
    float total = 0.f;
    for (int p = 0; p < pieces; ++p) total += part[((int64_t)p * pg.batch * n_kv_heads + row) * pg.max_ctx + i];
    const int64_t at = (int64_t)row * mass_stride + i;
    mass_out[at] = mass ? __builtin_fmaf(decay, mass[at], total) : total;
}

inline int64_t blocks_of(const kvs_shape *shape, int64_t max_ctx)
{
    const int keys = shape->dtype == KVS_F32 ? kWgKeys<KVS_F32> : kWgKeys<KVS_BF16>;
    return (max_ctx + keys - 1) / keys;
}

int pieces_of(const kvs_shape *shape, int64_t batch, int64_t max_ctx, int64_t n_new)
{
    const int64_t wgs = batch * shape->n_kv_heads * blocks_of(shape, max_ctx);
    const int64_t row_blocks = n_new * (shape->n_q_heads / shape->n_kv_heads) / (batch * kRows);
    if (wgs <= 0 || wgs >= 1024 || batch * shape->n_kv_heads > 65535) return 1;
    int64_t p = (2048 + wgs - 1) / wgs;
    if (p > row_blocks / 8) p = row_blocks / 8;
    if (p > kMaxPieces) p = kMaxPieces;
    return p < 1 ? 1 : (int)p;
}

template <int DTYPE, int D>
kvs_status launch(const kvs_shape *shape, const kvs_paged_cache *c, const Paged &pg, int64_t key_blocks, int pieces, const void *q, const float *lse, float scale, float decay,
                  const float *mass, float *mass_out, int64_t mass_stride, float *part, hipStream_t hs)
{
    hipLaunchKernelGGL((mass_paged_kernel<DTYPE, D>), dim3((unsigned)(key_blocks * pieces * pg.batch * shape->n_kv_heads)), dim3(kThreads), 0, hs, pg, shape->n_q_heads, shape->n_kv_heads,
                       (int)key_blocks, pieces, (const char *)c->k, (const char *)q, lse, scale * 1.4426950408889634f, decay, mass, mass_out, mass_stride, part);
    kvs_status st = check_launch("kvs_mass_paged");
    if (st != KVS_OK || pieces == 1) return st;
    hipLaunchKernelGGL(mass_join_kernel, dim3((unsigned)((pg.max_ctx + kThreads - 1) / kThreads), (unsigned)(pg.batch * shape->n_kv_heads)), dim3(kThreads), 0, hs, pg, shape->n_kv_heads,
                       pieces, part, decay, mass, mass_out, mass_stride);
    return check_launch("kvs_mass_paged(join)");
}

} // namespace

size_t mass_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx, int64_t n_new)
{
    if (check_shape(shape) != KVS_OK || batch <= 0 || max_ctx <= 0 || n_new <= 0) return 256;
    const int p = pieces_of(shape, batch, max_ctx, n_new);
    return p == 1 ? 256 : ((size_t)p * (size_t)batch * shape->n_kv_heads * (size_t)max_ctx * 4 + 255) / 256 * 256;
}

} // namespace kvs

extern "C" kvs_status kvs_mass_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                     const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new, const void *q_new, const float *lse, float scale,
                                     int32_t window, int32_t n_first, float decay, const float *mass, float *mass_out, int64_t mass_stride,
                                     void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace kvs;
    const char *me = "kvs_mass_paged";
    Paged pg;
    kvs_status st = check_paged(me, shape, cache, pages, &pg);
    if (st != KVS_OK || (st = check_new_tokens(me, shape, pages, cu_new, sel_pos, n_new, window, n_first, &pg)) != KVS_OK) return st;
    if (!isfinite(scale)) return fail(KVS_EINVAL, "%s: the scale is not finite", me);
    if (!isfinite(decay) || decay < 0.f) return fail(KVS_EINVAL, "%s: a decay of %g", me, (double)decay);
    if (mass_stride < pages->max_ctx) return fail(KVS_EINVAL, "%s: a mass stride of %lld for contexts of up to %lld", me, (long long)mass_stride, (long long)pages->max_ctx);
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(KVS_EINVAL, "%s: workspace must be 256-byte aligned", me);
    if (!workspace) workspace_bytes = 0;
    if (pages->batch == 0 || pg.max_ctx == 0) return KVS_OK;
    if (!mass_out) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    if (n_new > 0 && (!q_new || !lse)) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    if (!aligned16(q_new)) return fail(KVS_EINVAL, "%s: Q must be 16-byte aligned", me);
    const int64_t key_blocks = blocks_of(shape, pg.max_ctx);
    int pieces = pieces_of(shape, pg.batch, pg.max_ctx, n_new);
    const int64_t fit = (int64_t)(workspace_bytes / 4) / ((int64_t)pg.batch * shape->n_kv_heads * pg.max_ctx);
    if (pieces > fit) pieces = fit < 1 ? 1 : (int)fit;
    if (key_blocks * pieces * pg.batch * shape->n_kv_heads > kMostWgs) return fail(KVS_EINVAL, "%s: too many rows in one call", me);
    const bool wide = shape->head_dim == 128;
    hipStream_t hs = (hipStream_t)stream;
#define KVS_MP(DT, DD) launch<DT, DD>(shape, cache, pg, key_blocks, pieces, q_new, lse, scale, decay, mass, mass_out, mass_stride, (float *)workspace, hs)
    if (shape->dtype == KVS_F32) return wide ? KVS_MP(KVS_F32, 128) : KVS_MP(KVS_F32, 64);
    return wide ? KVS_MP(KVS_BF16, 128) : KVS_MP(KVS_BF16, 64);
#undef KVS_MP
}
