// kvs_attention_kv8: attention of selected rows, or of a decode step's single ones, over a cache held in 8 bits.
//
// Mathematics.  With codes k, v and their scales s_k, s_v for a block of tokens and a head, a row's output is
//     sum_i p_i s_v(i) v_i / sum_i p_i,   p_i = exp(scale s_k(i) (q . k_i) - max)
// Codes are bf16 numbers exactly, so they go to the matrix cores as they are: K's scale multiplies the score behind the
// first product, V's the weight before the second.  One pass over the keys with a running maximum and sum.
//
// Tiles.  A wave takes 32 rows (the query heads of one KV head flattened with the selected tokens, as in the bf16
// kernels) against tiles of 32 keys, S^T = K Q^T and O^T += V^T P^T, so that P stays in registers as the operand of the
// second product.  Tiles begin at multiples of 16 cache rows, whatever row a context begins at: each half of a tile then
// lies in one block, and its two scales are the same for all lanes.  What lies before a context, behind a row's position or
// behind the cache is masked.
//
// What bounds it with few rows, a decode step's, is the cache's bytes: 2 d a key and KV head.  So a workgroup's four
// waves take the same 32 rows and every fourth tile, each with LDS slots of its own that its loads go to directly
// (global to LDS, 16 bytes a lane, no registers), two tiles deep and without a barrier; at the end the waves meet in LDS.
// Launches of too few workgroups cut the key ranges into pieces, which a second kernel merges.  (One row of 8 query heads each over
// 131072 keys of 4 KV heads: 30 us and 4.4 for the merge, 4.5 TB/s in the first; 64 contexts of 4096 to 16384, 8 KV heads: 265 us,
// 5.1 TB/s.)
//
// With many rows the vector instructions do: a tile's 224 (e4m3: 64 conversions, 16 exponentials, 16 fused multiply-adds, and
// 8 comparisons more where it is masked; a wave's beginning and end in it, at 64 tiles a wave) beside 16 matrix instructions.  int8 has no
// conversion of its own and takes 128 more.  (800 rows of 32 query heads over 16000 keys: 153 to 172 us by box, 0.69 to 0.61 PFLOP/s of
// what the rows see; vector pipes busy 55 % of it, matrix pipes 27.)
//
// A lane's V operand is 8 keys of one channel, but a row of codes lies along the channels: the LDS reads that transpose
// bytes among 16 lanes give it those (64 bits a lane, from 8 rows of 16 bytes).
#include "cache8.h"
#include "attention.h"

#include <math.h>

namespace kvs {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kRows = 32;              // rows of a unit
constexpr int kKeys = 32;              // keys of a tile
constexpr int kAlign = 16;             // cache rows that tiles are aligned to: no block is shorter
constexpr float kSlack = 8.f;          // powers of two that a score may lie above its reference
constexpr int kMinPieceTiles = 4;      // tiles of a piece: one for each wave (with two, one row of 600 keys of 8 heads 9.9 us instead of 8.0, 4000 keys 9.9 and 8.6, in a graph)
constexpr int kMaxPieces = 512;
constexpr int64_t kMaxCutWgs = 2048;   // workgroups at most where key ranges are cut: four for every place on the chip

// The launch's requests.  Workgroup = (unit, KV head); a unit is a block of 32 rows of one request and one piece of its keys.
struct Table {
    int64_t ctx_off[kAttnMaxReq];
    int64_t sel0;                          // selected tokens before the launch
    int32_t ctx_len[kAttnMaxReq];
    int32_t unit_begin[kAttnMaxReq + 1];
    int32_t sel_begin[kAttnMaxReq + 1];    // selected tokens before the request, in this launch
    int32_t slot_begin[kAttnMaxReq];       // slots in the workspace before it: fewer than 32 kMaxCutWgs
    int32_t pieces[kAttnMaxReq];
    int32_t n_req, piece_tiles;
    int32_t interleaved;                   // unit u is unit u / n_req of request u % n_req, where that exists
};

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// a pair of codes (half `hi` of four) as a pair of bf16, exactly
template <int CODE, bool HI>
__device__ __forceinline__ uint32_t pair_of(uint32_t w)
{
    if constexpr (CODE == KVS_E4M3) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    } else {
        const float a = (float)(int8_t)((w >> (HI ? 16 : 0)) & 0xffu), b = (float)(int8_t)((w >> (HI ? 24 : 8)) & 0xffu);
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);   // whole numbers up to 128: 8 bits are enough
    }
}

// PARTS bf16 that add up to eight fp32 numbers each: to 16 of their bits with two, to all 24 with three.
template <int PARTS>
__device__ __forceinline__ void split(const float (&x)[8], u32x4_t (&part)[PARTS])
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack2(y[2 * i], y[2 * i + 1]);
            if (p == PARTS - 1) continue;
            y[2 * i] -= bf16_lo(w[i]);
            y[2 * i + 1] -= bf16_hi(w[i]);
        }
        part[p] = u32x4_t{w[0], w[1], w[2], w[3]};
    }
}

__device__ __forceinline__ float max_of_halves(float x)      // of lanes i and i + 32
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2_t *lds_i32x2;

// Byte `lane % 16` of eight rows of 16 bytes, the rows at which the lanes 16 i .. 16 i + 15 point, two lanes a row (at its halves).
__device__ __forceinline__ u32x2_t column8(const char *at)
{
    return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)at));
}

// The NaN that both NaN codes of e4m3 widen to (0xffc0) is the largest pattern there is: it becomes the negative of the largest number.
__device__ __forceinline__ u32x4_t numbers_of_bf16(u32x4_t v)
{
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(u32x4_t, __builtin_elementwise_min(__builtin_bit_cast(u16x8, v), (u16x8)(0xc3e0)));
}

typedef const __attribute__((address_space(4))) float *scalar_f32;    // read by all lanes at one address: scalar loads

// PARTS: bf16 numbers that a weight enters the second product as (bf16 only; fp32's are three)
template <int DTYPE, int CODE, int D, int PARTS>
__global__ __launch_bounds__(kThreads, 2) void attention8_kernel(
    const Table td, int n_q_heads, int n_kv_heads, int64_t n_rows, int block_log2,
    const uint8_t *__restrict__ k_codes, const uint8_t *__restrict__ v_codes, const float *__restrict__ k_scale, const float *__restrict__ v_scale,
    const void *__restrict__ q_sel, const int32_t *__restrict__ sel_pos, float scale_log2,
    void *__restrict__ out, float *__restrict__ lse_out, float *__restrict__ part_o, float4 *__restrict__ part_ml)
{
    constexpr int NQ = DTYPE == KVS_F32 ? 3 : 1;            // bf16 numbers that Q enters as
    constexpr int NP = DTYPE == KVS_F32 ? 3 : PARTS;        // ... and the weights
    constexpr int NDB = D / 32;                             // products of the second kind, channels a lane reads at once
    constexpr int CPR = D / 16;                             // 16-byte chunks of a row
    constexpr int RPL = kWave / CPR;                        // rows a load moves
    constexpr int NL = kKeys / RPL;                         // loads of a K or V tile
    constexpr int TILE_B = kKeys * D;
    constexpr bool V_EARLY = DTYPE == KVS_BF16 && CODE == KVS_E4M3;    // V is read beside the first product: 3% less time; int8's more conversions take 2% more so
    constexpr int WAVE_B = 4 * TILE_B;                      // two slots of (K, V); later the wave's 32 x D fp32 sums
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float4 ml_s[kWaves][kRows];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hf = lane >> 5, ln = lane & 31;

    const int g = blockIdx.x % n_kv_heads;
    const int unit = (int)(blockIdx.x / n_kv_heads);
    const int b = td.interleaved ? unit % td.n_req : request_of(td.unit_begin, td.n_req, unit);
    const int in_req = td.interleaved ? unit / td.n_req : unit - td.unit_begin[b];
    if (in_req >= td.unit_begin[b + 1] - td.unit_begin[b]) return;
    const int pieces = td.pieces[b], row_blocks = (td.unit_begin[b + 1] - td.unit_begin[b]) / pieces;
    // A piece's row blocks run side by side, which share its keys in L2, and the last rows, which see most, begin.
    const int piece = in_req / row_blocks, row_block = row_blocks - 1 - in_req % row_blocks;
    const int grp = n_q_heads / n_kv_heads;
    const int ctx_len = td.ctx_len[b];
    const int rows = (td.sel_begin[b + 1] - td.sel_begin[b]) * grp;      // the host keeps this below 2^31
    const int64_t sel_lo = td.sel0 + td.sel_begin[b];

    // ---- this lane's row (both half-waves hold the same 32) ------------------------------------------------
    const int rq = min(row_block * kRows + ln, rows - 1);
    const int t_sel = rq / grp, hh = rq - t_sel * grp;
    int pos = sel_pos[sel_lo + t_sel];
    // keys are counted from the 16-row boundary at or before the context: x = key + shift
    const int shift = (int)(td.ctx_off[b] & (kAlign - 1));
    const int64_t row0 = td.ctx_off[b] - shift;
    const int64_t t_lo = (int64_t)piece * td.piece_tiles, t_most = t_lo + td.piece_tiles;
    // the wave's tiles are t_lo + wave + kWaves i, as many as lie below x (and the piece's end)
    auto tiles_below = [&](int64_t x) -> int {
        const int64_t end = min((x + kKeys - 1) / kKeys, t_most);
        return (int)max((int64_t)0, (end - t_lo - wave + kWaves - 1) / kWaves);
    };

    // ---- Q as the B operand: k-step 2i + s takes channels 32i + 16hf + 8s .. +7, as the K rows are read below.  A negative
    // scale's sign goes into Q, so that the largest score is the largest product's -------------------------------
    const bool negative = scale_log2 < 0.f;
    const float scale_abs = fabsf(scale_log2);
    bf16x8 qreg[NQ][D / 16];
    {
        const int64_t at = ((sel_lo + t_sel) * n_q_heads + g * grp + hh) * (int64_t)D + 16 * hf;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const int c = 32 * (ks >> 1) + 8 * (ks & 1);
            if constexpr (DTYPE == KVS_BF16) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t *>((const uint16_t *)q_sel + at + c);
                qreg[0][ks] = as_bf16x8(w ^ (negative ? 0x80008000u : 0u));
            } else {
                const float4 lo = *reinterpret_cast<const float4 *>((const float *)q_sel + at + c), hi = *reinterpret_cast<const float4 *>((const float *)q_sel + at + c + 4);
                float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = negative ? -x[j] : x[j];
                u32x4_t part[3];
                split(x, part);
#pragma unroll
                for (int p = 0; p < NQ; ++p) qreg[p][ks] = as_bf16x8(part[p]);
            }
        }
    }

    // ---- staging ------------------------------------------------------------------------------------------------
    // A load moves RPL rows of the tile, 16 bytes a lane, to consecutive LDS.  Chunk c of row r lies at position c ^ swz(r):
    // eight (four) neighbouring rows then use all banks where a chunk is read down the rows.
    char *const my_lds = lds + wave * WAVE_B;
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)my_lds);
    const uint32_t row_bytes = (uint32_t)n_kv_heads * D;
    auto swz = [](int r) { return D == 128 ? (r & 7) : ((r >> 1) & 3); };
    const int st_row = lane / CPR, st_chunk = (lane % CPR) ^ swz(st_row);
    const uint32_t st_off = (uint32_t)st_row * row_bytes + (uint32_t)st_chunk * 16u;
    // Written by hand: issued through the compiler's builtin, every later LDS read would wait for all loads in flight.  M0 holds
    // the LDS address of lane 0; the nop is the wait state that a write to M0 needs before such a load.
    auto load_1k = [&](uint32_t dst, uint32_t off, const uint8_t *base) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst), "v"(off), "s"(base) : "memory");
    };
    // Rows and scales of the wave's tiles lie at constant steps: kWaves tiles are 128 rows, a multiple of every block.
    const int64_t first_row = row0 + (t_lo + wave) * kKeys;
    auto stage = [&](int64_t first, int slot) {
        const int64_t at = (first * n_kv_heads + g) * D;
        const uint32_t dst = lds_base + (uint32_t)slot * (2 * TILE_B);
        if (first + kKeys <= n_rows) {
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                load_1k(dst + j * 1024, st_off + (uint32_t)(j * RPL) * row_bytes, k_codes + at);
                load_1k(dst + TILE_B + j * 1024, st_off + (uint32_t)(j * RPL) * row_bytes, v_codes + at);
            }
        } else {                                            // the cache ends inside: its last row again and again
            const int last = (int)(n_rows - 1 - first);
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const uint32_t off = (uint32_t)min(st_row + j * RPL, last) * row_bytes + (uint32_t)st_chunk * 16u;
                load_1k(dst + j * 1024, off, k_codes + at);
                load_1k(dst + TILE_B + j * 1024, off, v_codes + at);
            }
        }
    };
    static_assert(kWaves * kKeys % 128 == 0, "a multiple of the largest block");
    struct Scales { float k[2], v[2]; };
    const int64_t scale_step = ((int64_t)(kWaves * kKeys) >> block_log2) * n_kv_heads;
    const int64_t scale_at = (first_row >> block_log2) * n_kv_heads + g;
    const int second_half = (int)((first_row + kAlign) >> block_log2) != (int)(first_row >> block_log2) ? n_kv_heads : 0;
    const scalar_f32 ks_p = (scalar_f32)(uintptr_t)k_scale + scale_at, vs_p = (scalar_f32)(uintptr_t)v_scale + scale_at;
    auto scales_of = [&](int i, int64_t first) {
        const int64_t lo = i * scale_step, hi = lo + (first + kAlign < n_rows ? second_half : 0);
        return Scales{{ks_p[lo], ks_p[hi]}, {vs_p[lo], vs_p[hi]}};
    };

    // The first two tiles are asked for before anybody knows how far the rows see: as if they saw the whole context.
    const int whole = tiles_below(ctx_len > 0 ? (int64_t)ctx_len + shift : 0);
    if (whole > 0) stage(first_row, 0);
    if (whole > 1) stage(first_row + kWaves * kKeys, 1);
    Scales next = {};
    if (whole > 0) next = scales_of(0, first_row);
    pos = pos < 0 ? -1 : min(pos, ctx_len - 1);
    int pmin = pos, pmax = pos;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        pmin = min(pmin, __shfl_xor(pmin, o));
        pmax = max(pmax, __shfl_xor(pmax, o));
    }
    pmin = __builtin_amdgcn_readfirstlane(pmin);
    pmax = __builtin_amdgcn_readfirstlane(pmax);
    const int xpos = pos < 0 ? -1 : pos + shift;            // last x that the row sees; the first is `shift`
    const int mine = tiles_below(pmax < 0 ? 0 : (int64_t)pmax + shift + 1);

    // ---- running state ------------------------------------------------------------------------------------------
    floatx16 o_acc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[db][r] = 0.f;
    float m_run = kLowest;     // reference of the weights: a former maximum of the scores times log2 e, the same in both half-waves
    float l_run = 0.f;         // this half-wave's share of the sum of weights
    float l_rnd = 0.f;         // the same of the weights as the second product sees them (bf16)
    // K row of matrix row ln: bits 2 and 3 swapped, so that accumulator entry r is key 16 (r >> 3) + 8 hf + (r & 7)
    const int krow = (ln & ~12) | ((ln & 4) << 1) | ((ln & 8) >> 1);

    int x0 = (int)((t_lo + wave) * kKeys);                   // (contexts are shorter than 2^31)
    int64_t tile_row = first_row;
    for (int i = 0; i < mine; ++i, x0 += kWaves * kKeys, tile_row += kWaves * kKeys) {
        const Scales sc = next;
        if (i + 1 < mine) next = scales_of(i + 1, tile_row + kWaves * kKeys);
        // this tile has landed; the next one's loads may still be on their way
        if (i + 1 < mine || (i == 0 && whole > 1)) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * NL) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        char *const kt = my_lds + (i & 1) * (2 * TILE_B);
        char *const vt = kt + TILE_B;
        const bool masked = x0 < shift || x0 + kKeys - 1 > pmin + shift || pmin < 0;

        // Memory that was never stored to may hold NaN codes: in rows that are masked, and in blocks of scale 0.  Masked scores
        // are replaced whatever they are, and V's codes become numbers behind their conversion.
        if (CODE == KVS_E4M3 && (sc.k[0] == 0.f || sc.k[1] == 0.f)) {
#pragma unroll
            for (int e = 0; e < TILE_B / 1024; ++e) {
                u32x4_t *w = reinterpret_cast<u32x4_t *>(kt) + e * kWave + lane;
                u32x4_t c = *w;
                c.x = numbers_only(c.x); c.y = numbers_only(c.y); c.z = numbers_only(c.z); c.w = numbers_only(c.w);
                *w = c;
            }
        }
        u32x4_t va[2][NDB];                                  // of channel 32 db + ln, keys 16 a + 8 hf .. + 7
        auto v_operands = [&](int a) {
            const int key = 16 * a + 8 * hf + ((ln & 15) >> 1);          // the row that the lane points at, for the lanes of its 16
            const char *from = vt + key * D + (ln & 1) * 8;
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
                const u32x2_t w = column8(from + ((2 * db + (ln >> 4)) ^ swz(key)) * 16);
                va[a][db] = u32x4_t{pair_of<CODE, false>(w.x), pair_of<CODE, true>(w.x), pair_of<CODE, false>(w.y), pair_of<CODE, true>(w.y)};
            }
        };
        floatx16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t *>(kt + krow * D + ((2 * c + hf) ^ swz(krow)) * 16);
            const u32x4_t lo = {pair_of<CODE, false>(w.x), pair_of<CODE, true>(w.x), pair_of<CODE, false>(w.y), pair_of<CODE, true>(w.y)};
            const u32x4_t hi = {pair_of<CODE, false>(w.z), pair_of<CODE, true>(w.z), pair_of<CODE, false>(w.w), pair_of<CODE, true>(w.w)};
#pragma unroll
            for (int p = 0; p < NQ; ++p) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(lo), qreg[p][2 * c], s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(hi), qreg[p][2 * c + 1], s, 0, 0, 0);
            }
        }
        if constexpr (V_EARLY) { v_operands(0); v_operands(1); }
        // (a broken block's V makes the scores NaN too, as the widened contexts' K does: sums and log-sum-exps then say so)
        float f[2] = {__builtin_fmaf(sc.v[0], 0.f, sc.k[0] * scale_abs), __builtin_fmaf(sc.v[1], 0.f, sc.k[1] * scale_abs)};
        const int first = shift - x0 - 8 * hf, last = xpos - x0 - 8 * hf;     // entries 16 (r >> 3) + (r & 7) from `first` to `last` are seen
        auto entry = [](int r) { return 16 * (r >> 3) + (r & 7); };
        if (masked) {
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                if (!(f[a] > 0.f && f[a] < INFINITY)) {      // 0 or NaN times the -infinity of what is masked
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[8 * a + j] *= f[a];
                    f[a] = 1.f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) s[8 * a + j] = entry(8 * a + j) <= last ? s[8 * a + j] : -INFINITY;
            }
            if (x0 < shift) {                                // a context's first tile
#pragma unroll
                for (int r = 0; r < 8; ++r) s[r] = entry(r) >= first ? s[r] : -INFINITY;
            }
        }
        float mx_tile = -INFINITY;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            float mx = s[8 * a];
#pragma unroll
            for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[8 * a + j]);
            mx_tile = fmaxf(mx_tile, mx * f[a]);
        }
        mx_tile = max_of_halves(mx_tile);
        // The reference that weights are relative to moves only once a score is kSlack above it (in powers of two): weights of up
        // to 2^kSlack lose nothing, and sums are seldom scaled behind a row's first tiles.
        if (__builtin_amdgcn_ballot_w64(mx_tile > m_run + kSlack) != 0) {
            const float m_new = fmaxf(m_run, mx_tile), corr = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= corr;
            l_rnd *= corr;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o_acc[db][r] *= corr;
        }
        u32x4_t pop[2][NP];
        float psum = 0.f, rsum = 0.f;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            float y[8], group = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * a + j], f[a], -m_run));
                group += p;
                y[j] = p * sc.v[a];
            }
            if (masked && !(fabsf(sc.v[a]) < INFINITY)) {    // 0 times a broken block's scale
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = entry(8 * a + j) <= last && entry(8 * a + j) >= first ? y[j] : 0.f;
            }
            psum += group;
            if constexpr (NP == 1) {
                // The normaliser is made of the rounded weights: numerator and denominator then carry the same rounding, and a
                // row that one key dominates returns that key's V to within the output's own rounding.
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                float rounded = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = pack2(y[2 * j], y[2 * j + 1]);
                    pop[a][0][j] = w;
                    rounded = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), rounded, false);
                }
                // (scales below 2^-80 would bring weights below what bf16 holds)
                rsum += sc.v[a] > 8.271806e-25f ? rounded * __builtin_amdgcn_rcpf(sc.v[a]) : group;
            } else {
                split(y, pop[a]);
            }
        }
        l_run += psum;
        l_rnd += rsum;

        const bool dirty = CODE == KVS_E4M3 && (masked || sc.v[0] == 0.f || sc.v[1] == 0.f);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            if constexpr (!V_EARLY) v_operands(a);
            if (dirty) {
#pragma unroll
                for (int db = 0; db < NDB; ++db) va[a][db] = numbers_of_bf16(va[a][db]);
            }
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int p = 0; p < NP; ++p) o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(va[a][db]), as_bf16x8(pop[a][p]), o_acc[db], 0, 0, 0);
        }
        if (i + 2 < mine) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // what lay in the slot has been read
            stage(tile_row + 2 * kWaves * kKeys, i & 1);
        }
    }

    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // tiles that no row sees may still be on their way into LDS

    // ---- the waves meet --------------------------------------------------------------------------------------------
    {
        const float l = l_run + __shfl_xor(l_run, 32), lr = l_rnd + __shfl_xor(l_rnd, 32);
        if (hf == 0) ml_s[wave][ln] = make_float4(m_run, l, NP == 1 ? lr : l, 0.f);
    }
    __syncthreads();
    {
        float top = ml_s[0][ln].x;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml_s[w][ln].x);
        const float f = __builtin_amdgcn_exp2f(m_run - top);
        float *mine_o = reinterpret_cast<float *>(my_lds) + ln * D;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c4 = 8 * db + 2 * q + hf;          // channels 4 c4 .. + 3: at place c4 ^ row, so that rows use different banks
                *reinterpret_cast<float4 *>(mine_o + 4 * (c4 ^ (ln & (D / 4 - 1)))) =
                    make_float4(o_acc[db][4 * q] * f, o_acc[db][4 * q + 1] * f, o_acc[db][4 * q + 2] * f, o_acc[db][4 * q + 3] * f);
            }
    }
    __syncthreads();
    constexpr int CPT = D / 8;                               // channels a thread stores
    const int row = tid >> 3, part = tid & 7;
    const int row_q = row_block * kRows + row;
    if (row_q >= rows) return;
    float top = kLowest, l = 0.f, lr = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml_s[w][row].x);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float4 x = ml_s[w][row];
        const float f = __builtin_amdgcn_exp2f(x.x - top);
        l += x.y * f;
        lr += x.z * f;
    }
    float o[CPT];
#pragma unroll
    for (int c = 0; c < CPT; ++c) o[c] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float *from = reinterpret_cast<const float *>(lds + w * WAVE_B) + row * D;
#pragma unroll
        for (int k = 0; k < CPT / 4; ++k) {
            const float4 y = *reinterpret_cast<const float4 *>(from + 4 * ((CPT / 4 * part + k) ^ (row & (D / 4 - 1))));
            o[4 * k] += y.x; o[4 * k + 1] += y.y; o[4 * k + 2] += y.z; o[4 * k + 3] += y.w;
        }
    }
    const int t2 = row_q / grp, h2 = row_q - t2 * grp;
    const int64_t at = (sel_lo + t2) * n_q_heads + g * grp + h2;
    if (pieces > 1) {
        const int64_t slot = td.slot_begin[b] + ((int64_t)t2 * n_q_heads + g * grp + h2) * pieces + piece;
        if (part == 0) part_ml[slot] = make_float4(top, l, lr, 0.f);
        if (l != 0.f) {                                      // (the merge passes over a piece without keys)
            float4 *dst = reinterpret_cast<float4 *>(part_o + slot * D + part * CPT);
#pragma unroll
            for (int c = 0; c < CPT / 4; ++c) dst[c] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
        }
        return;
    }
    const float inv = l != 0.f ? 1.f / lr : 0.f;
#pragma unroll
    for (int c = 0; c < CPT; ++c) o[c] = l != 0.f ? o[c] * inv : 0.f;
    if constexpr (DTYPE == KVS_BF16) {
        uint4 *dst = reinterpret_cast<uint4 *>((uint16_t *)out + at * D + part * CPT);
#pragma unroll
        for (int c = 0; c < CPT / 8; ++c)
            dst[c] = make_uint4(pack2(o[8 * c], o[8 * c + 1]), pack2(o[8 * c + 2], o[8 * c + 3]), pack2(o[8 * c + 4], o[8 * c + 5]), pack2(o[8 * c + 6], o[8 * c + 7]));
    } else {
        float4 *dst = reinterpret_cast<float4 *>((float *)out + at * D + part * CPT);
#pragma unroll
        for (int c = 0; c < CPT / 4; ++c) dst[c] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
    }
    if (lse_out && part == 0) lse_out[at] = l != 0.f ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// out = sum_p w_p O_p / sum_p w_p l_p with w_p = 2^(m_p - max m).  A workgroup takes 32 channels of one row: its threads make the
// pieces' weights once, into LDS, then groups of 8 threads take every 32nd piece, four channels a thread, and meet by shuffles and in LDS.
// (A wave a row, piece after piece, spent its time on one round trip to memory after the other: 256 pieces 80 us; a workgroup
// for all channels of a row took 5.7 us for 74 pieces of 32 rows, this 4.5; 114 pieces of 32 rows 4.4.)
template <int DTYPE, int D>
__global__ __launch_bounds__(kThreads) void merge8_kernel(const Table td, int n_q_heads, const float *__restrict__ part_o,
                                                          const float4 *__restrict__ part_ml, void *__restrict__ out, float *__restrict__ lse_out)
{
    constexpr int kLanes = 8, kGroups = kThreads / kLanes;
    __shared__ float weight[kMaxPieces];
    __shared__ float meet[3][kWaves];
    __shared__ float4 sum_s[kWaves][kLanes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int item = (int)blockIdx.x;
    const int b = request_of(td.sel_begin, td.n_req, item / n_q_heads);
    const int pieces = td.pieces[b];
    if (pieces <= 1) return;                                 // stored as it is by its only workgroup
    const int64_t local = item - (int64_t)td.sel_begin[b] * n_q_heads;
    const int64_t slot = td.slot_begin[b] + local * pieces;
    static_assert(kMaxPieces == 2 * kThreads, "two records a thread");
    float4 x[2];
    float top = kLowest;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = tid + i * kThreads;
        x[i] = p < pieces ? part_ml[slot + p] : make_float4(kLowest, 0.f, 0.f, 0.f);
        top = fmaxf(top, x[i].x);
    }
    top = wave_max(top);
    if (lane == 0) meet[0][wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, meet[0][w]);
    float l = 0.f, lr = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float f = __builtin_amdgcn_exp2f(x[i].x - top);
        l += x[i].y * f;
        lr += x[i].z * f;
        if (tid + i * kThreads < pieces) weight[tid + i * kThreads] = x[i].y != 0.f ? f : -1.f;      // (-1: a piece without keys has left no sums)
    }
    l = wave_sum(l);
    lr = wave_sum(lr);
    if (lane == 0) { meet[1][wave] = l; meet[2][wave] = lr; }
    __syncthreads();
    l = (meet[1][0] + meet[1][1]) + (meet[1][2] + meet[1][3]);
    lr = (meet[2][0] + meet[2][1]) + (meet[2][2] + meet[2][3]);
    const int c = (int)blockIdx.y * kLanes + tid % kLanes;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4 *from = reinterpret_cast<const float4 *>(part_o + slot * D) + c;
#pragma unroll 4
    for (int p = tid / kLanes; p < pieces; p += kGroups) {
        const float f = weight[p];
        const float4 y = f >= 0.f ? from[(int64_t)p * (D / 4)] : make_float4(0.f, 0.f, 0.f, 0.f);
        const float g = fmaxf(f, 0.f);
        o.x += g * y.x; o.y += g * y.y; o.z += g * y.z; o.w += g * y.w;
    }
#pragma unroll
    for (int m = kLanes; m < kWave; m <<= 1) {
        o.x += __shfl_xor(o.x, m); o.y += __shfl_xor(o.y, m); o.z += __shfl_xor(o.z, m); o.w += __shfl_xor(o.w, m);
    }
    if (lane < kLanes) sum_s[wave][lane] = o;
    __syncthreads();
    if (tid >= kLanes) return;
#pragma unroll
    for (int i = 1; i < kWaves; ++i) {
        const float4 y = sum_s[i][lane];
        o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
    }
    const int64_t at = td.sel0 * n_q_heads + item;
    const float inv = 1.f / lr;
    if (l != 0.f) { o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv; }
    else o = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (DTYPE == KVS_BF16) *reinterpret_cast<uint2 *>((uint16_t *)out + at * D + 4 * c) = make_uint2(pack2(o.x, o.y), pack2(o.z, o.w));
    else *reinterpret_cast<float4 *>((float *)out + at * D + 4 * c) = o;
    if (lse_out && c == 0) lse_out[at] = l != 0.f ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// The same where no row has more than kFewPieces: D / 4 threads a row, four channels a thread, all pieces asked for at once.
constexpr int kFewPieces = 16;
template <int DTYPE, int D>
__global__ __launch_bounds__(kThreads) void merge8_rows_kernel(const Table td, int n_items, int n_q_heads, const float *__restrict__ part_o,
                                                               const float4 *__restrict__ part_ml, void *__restrict__ out, float *__restrict__ lse_out)
{
    constexpr int kLanes = D / 4;
    const int c = threadIdx.x % kLanes;
    const int item = (int)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    if (item >= n_items) return;
    const int b = request_of(td.sel_begin, td.n_req, item / n_q_heads);
    const int pieces = td.pieces[b];
    if (pieces <= 1) return;
    const int64_t local = item - (int64_t)td.sel_begin[b] * n_q_heads;
    const int64_t slot = td.slot_begin[b] + local * pieces;
    const float4 *from = reinterpret_cast<const float4 *>(part_o + slot * D) + c;
    float4 x[kFewPieces], y[kFewPieces];
    float top = kLowest;
#pragma unroll
    for (int p = 0; p < kFewPieces; ++p) {
        x[p] = p < pieces ? part_ml[slot + p] : make_float4(kLowest, 0.f, 0.f, 0.f);
        y[p] = p < pieces ? from[(int64_t)p * kLanes] : make_float4(0.f, 0.f, 0.f, 0.f);
        top = fmaxf(top, x[p].x);
    }
    float l = 0.f, lr = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int p = 0; p < kFewPieces; ++p) {
        const float f = __builtin_amdgcn_exp2f(x[p].x - top);
        l += x[p].y * f;
        lr += x[p].z * f;
        if (x[p].y != 0.f) { o.x += f * y[p].x; o.y += f * y[p].y; o.z += f * y[p].z; o.w += f * y[p].w; }       // (a piece without keys has left no sums)
    }
    const int64_t at = td.sel0 * n_q_heads + item;
    const float inv = 1.f / lr;
    if (l != 0.f) { o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv; }
    else o = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (DTYPE == KVS_BF16) *reinterpret_cast<uint2 *>((uint16_t *)out + at * D + 4 * c) = make_uint2(pack2(o.x, o.y), pack2(o.z, o.w));
    else *reinterpret_cast<float4 *>((float *)out + at * D + 4 * c) = o;
    if (lse_out && c == 0) lse_out[at] = l != 0.f ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

inline size_t slot_bytes(int d) { return (size_t)d * sizeof(float) + sizeof(float4); }

// How a launch's key ranges are cut: pieces of `piece_tiles` tiles (0: not at all).
struct Plan { int64_t piece_tiles, slots; };

inline int64_t tiles_of(int64_t ctx_len) { return (ctx_len + kAlign - 1 + kKeys - 1) / kKeys; }    // wherever in a block it begins
inline int64_t blocks_of(int64_t n_sel, int grp) { return (n_sel * grp + kRows - 1) / kRows; }

// The piece with the least estimated time, of those whose slots the workspace holds.  In microseconds, as measured: a workgroup
// takes kAlone for a tile, kTile beside a second one on its CU, and kStart besides; the caches are read at kBytes a microsecond,
// row blocks of the same keys from L2, and an eighth slower by one workgroup a CU; reading and computing hide each other less
// the closer they are; behind the average workgroup's end the longest go on by themselves; a merge costs its launch (2 in a
// full queue, 5 where the device waits for the host) and its slots, written and read.  Rows of several blocks are taken to be
// spread over their context, and to see half of it.
Plan plan_pieces(const kvs_shape *shape, int32_t n_req, const int64_t *ctx_len, const int64_t *cu_sel, size_t workspace_bytes)
{
    constexpr double kPlaces = 512, kAlone = 0.32, kTile = 0.38, kStart = 4.0, kBytes = 4.9e6, kMerge = 5.0, kSlotBytes = 2e6;
    const int grp = shape->n_q_heads / shape->n_kv_heads, hk = shape->n_kv_heads;
    const double tile_bytes = 2.0 * kKeys * shape->head_dim;
    double wgs1 = 0, load = 0, bytes = 0;
    int64_t longest = 0;
    for (int32_t b = 0; b < n_req; ++b) {
        const int64_t n = cu_sel[b + 1] - cu_sel[b], t = tiles_of(ctx_len[b]);
        if (n == 0) continue;
        const double nb = (double)blocks_of(n, grp), tiles = (double)t;
        wgs1 += nb * hk;
        load += (nb > 1 ? (nb + 1) / 2 : 1) * hk * tiles;
        bytes += hk * tiles * tile_bytes;
        if (t > longest) longest = t;
    }
    if (wgs1 > (double)kMaxCutWgs || longest <= kMinPieceTiles) return {0, 0};
    Plan best = {0, 0};
    double best_us = 1e30;
    for (int64_t cuts = 1; cuts <= kMaxPieces; cuts += (cuts + 3) / 4) {
        int64_t piece = ((longest + cuts - 1) / cuts + kWaves - 1) / kWaves * kWaves;
        if (piece < kMinPieceTiles) piece = kMinPieceTiles;
        int64_t slots = 0;
        double wgs = 0, busy = 0;                            // ... and those of them with keys
        for (int32_t b = 0; b < n_req; ++b) {
            const int64_t n = cu_sel[b + 1] - cu_sel[b];
            if (n == 0) continue;
            const int64_t p = (tiles_of(ctx_len[b]) + piece - 1) / piece, nb = blocks_of(n, grp);
            if (p > 1) slots += n * shape->n_q_heads * p;
            wgs += (double)(nb * (p > 1 ? p : 1) * hk);
            busy += p > 1 ? (nb > 1 ? 0.5 * (double)((p + 1) * nb) : (double)p) * hk : (double)(nb * hk);
        }
        if (cuts > 1 && ((size_t)slots * slot_bytes(shape->head_dim) > workspace_bytes || wgs > (double)kMaxCutWgs)) break;
        const double places = busy < kPlaces ? busy : kPlaces;
        const double second = busy <= kPlaces / 2 ? 0 : (places - kPlaces / 2) / (kPlaces / 2);         // CUs with a second workgroup
        const double reading = bytes / (kBytes * (0.88 + 0.12 * second)), computing = load / places * (kAlone + (kTile - kAlone) * second);
        const double tail = busy <= kPlaces ? (double)piece - load / busy : (double)piece * (slots ? 0.35 : 0.25);
        double us = cbrt(reading * reading * reading + computing * computing * computing) + (tail > 0 ? tail * kAlone : 0) + kStart * (busy > kPlaces ? busy / kPlaces : 1);
        if (slots) us += kMerge + 2 * (double)slots * (double)slot_bytes(shape->head_dim) / kSlotBytes;
        if (us < best_us) {
            best_us = us;
            best = slots ? Plan{piece, slots} : Plan{0, 0};
        }
        if (piece == kMinPieceTiles) break;
    }
    return best;
}

// ---- many rows a key: a bf16 copy --------------------------------------------------------------------------------
// With hundreds of rows a key and KV head the matrix cores could bound the call, but above every wave widens all keys that it
// multiplies with: 64 vector instructions (int8: 192) beside the 16 matrix products of a tile, for 32 rows.  Such
// launches widen the contexts once, into the workspace, and go to the bf16 kernel of 256 rows (attention_mfma2.hip).  K
// goes there as its codes and V as codes times the power of two below its scale, which bf16 holds exactly; for every 16 rows
// and KV head there is a factor of the scores, and the rest of V's scale, in [1, 2), as a summand of the exponents, with its
// inverse for the sums of weights (attn_mfma2_kernel's SCALED).
constexpr int kCopyThreads = 256;

// A normal number's significand, in [1, 2); 1 for all others.
__device__ __forceinline__ float rest_of_scale(float s)
{
    const float a = fabsf(s);
    return a >= kLeastScale && a < INFINITY ? __uint_as_float((__float_as_uint(s) & 0x7fffffu) | 0x3f800000u) : 1.f;
}

// The rows that the requests of a launch see, as ranges that share no row (requests may see the same rows), and the copy holds one range
// behind the other.
struct CopyRanges {
    int64_t row[kAttnMaxReq];              // first row of range i, a multiple of 16
    int32_t begin[kAttnMaxReq + 1];        // groups of 16 rows before it in the copy
    int32_t n;
};

template <int CODE>
__global__ __launch_bounds__(kCopyThreads) void copy8_kernel(const CopyRanges cr, int n_kv_heads, int64_t n_rows, int block_log2,
                                                             const uint4 *__restrict__ k_codes, const uint4 *__restrict__ v_codes,
                                                             const float *__restrict__ k_scale, const float *__restrict__ v_scale, float scale_log2,
                                                             uint4 *__restrict__ k_out, uint4 *__restrict__ v_out, float4 *__restrict__ factors, int64_t factor_stride)
{
    constexpr int kChunks = 128 / 16;
    const int64_t group = blockIdx.x;                                                   // of the copy
    const int b = request_of(cr.begin, cr.n, (int)group);
    const int64_t row0 = cr.row[b] + (group - cr.begin[b]) * kAlign;                    // the workgroup's 16 rows: one block of scales
    const int64_t scales = (min(row0, n_rows - 1) >> block_log2) * n_kv_heads;
    const int rows = (int)min((int64_t)kAlign, n_rows - row0);                          // (none where only the factors of a tile's second half are wanted)
    for (int g = threadIdx.x; g < n_kv_heads; g += kCopyThreads) {
        // (positive and finite, whatever the scale: a block that stands for zeros has codes of 0, a broken one NaN in K)
        const float f = k_scale[scales + g] * scale_log2;
        const float m = rest_of_scale(v_scale[scales + g]);
        factors[g * factor_stride + group] = make_float4(f >= 7.888609e-31f && f < INFINITY ? f : 7.888609e-31f, __log2f(m), 1.f / m, 0.f);
    }
    const int per_row = n_kv_heads * kChunks;
    for (int e = threadIdx.x; e < rows * per_row; e += kCopyThreads) {
        const int c = e % per_row;
        const int64_t from = row0 * per_row + e, to = (group * kAlign * per_row + e) * 2;
        const float ks = k_scale[scales + c / kChunks], vs = v_scale[scales + c / kChunks];
        const float v_by = rest_of_scale(vs) == 1.f ? vs : __uint_as_float(__float_as_uint(vs) & 0xff800000u);
        const uint4 k = stream_load16(k_codes + from), v = stream_load16(v_codes + from);
        const bool broken = !(fabsf(ks) < INFINITY) || !(fabsf(vs) < INFINITY);
        const uint32_t kw[4] = {k.x, k.y, k.z, k.w}, vw[4] = {v.x, v.y, v.z, v.w};
        uint32_t ko[8], vo[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t kc = CODE == KVS_E4M3 ? numbers_only(kw[i]) : kw[i], vc = CODE == KVS_E4M3 ? numbers_only(vw[i]) : vw[i];
            ko[2 * i] = broken ? 0x7fc07fc0u : ks > 0.f ? pair_of<CODE, false>(kc) : 0u;
            ko[2 * i + 1] = broken ? 0x7fc07fc0u : ks > 0.f ? pair_of<CODE, true>(kc) : 0u;
            float x[4];
            widen_codes<CODE>(vc, x);
            vo[2 * i] = broken ? 0u : pack2(x[0] * v_by, x[1] * v_by);
            vo[2 * i + 1] = broken ? 0u : pack2(x[2] * v_by, x[3] * v_by);
        }
        k_out[to] = make_uint4(ko[0], ko[1], ko[2], ko[3]);
        k_out[to + 1] = make_uint4(ko[4], ko[5], ko[6], ko[7]);
        v_out[to] = make_uint4(vo[0], vo[1], vo[2], vo[3]);
        v_out[to + 1] = make_uint4(vo[4], vo[5], vo[6], vo[7]);
    }
}

// The bf16 kernel takes a negative position for 0: the rows of tokens that see nothing become 0 here.  A wave a token.
__global__ __launch_bounds__(kThreads) void empty_rows_kernel(int64_t n_sel, int n_q_heads, const int32_t *__restrict__ sel_pos, uint4 *__restrict__ out,
                                                              float *__restrict__ lse_out)
{
    const int64_t s = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (s >= n_sel || sel_pos[s] >= 0) return;
    const int lane = threadIdx.x & 63;
    for (int e = lane; e < n_q_heads * 16; e += 64) out[s * n_q_heads * 16 + e] = make_uint4(0u, 0u, 0u, 0u);
    for (int h = lane; lse_out && h < n_q_heads; h += 64) lse_out[s * n_q_heads + h] = -INFINITY;
}

constexpr int64_t kCopyMinRows = 7373;     // selected rows over all query heads: 48 tiles of 256, 0.6 full, as the bf16 kernel asks for
constexpr int64_t kCopyPad = 8;            // factors behind the last row's: what a step ahead asks for
inline size_t copy_bytes(const kvs_shape *shape, int64_t groups)
{
    return (size_t)(groups * kAlign * shape->n_kv_heads * 128 * 4 + (groups + kCopyPad) * shape->n_kv_heads * (int64_t)sizeof(float4) + 512);
}
// Groups that the ranges of a launch have at most, for requests of `rows` rows together: each ends with a part of one, and one more.
inline int64_t copy_groups(int32_t batch, int64_t rows)
{
    const int64_t n = batch < 1 ? 1 : batch < kAttnMaxReq ? batch : kAttnMaxReq;
    return (rows + kAlign - 1) / kAlign + 2 * n;
}

// Whether a copy for the bf16 kernel is worth its bytes.  Measured, of what rows in the middle of their contexts take: the kernel above
// 0.66 PFLOP/s of e4m3 and 0.52 of int8, the bf16 kernel 1.05, the copy 6 bytes an element of K and V at 4.5 TB/s, and 55 us
// for two more launches and the bf16 kernel's larger tiles at its end.  (800 rows of 16000, 32 heads: 172 us here, 183 through a
// copy; 900 of 30000 339 and 325; 3 x 500 of 8000 157 and 179; 4424 of 32768 1552 and 1150.)
bool bf16_copy_pays(const kvs_shape *shape, const kvs_cache8 *cache, int32_t n_req, const int64_t *ctx_off, const int64_t *ctx_len, const int64_t *cu_sel, float scale)
{
    if (shape->dtype != KVS_BF16 || shape->head_dim != 128 || !(scale > 0.f)) return false;
    const int64_t rows = (cu_sel[n_req] - cu_sel[0]) * shape->n_q_heads;
    if (rows < kCopyMinRows) return false;
    double flops = 0, bytes = 0;
    for (int32_t b = 0; b < n_req; ++b) {
        const int64_t n = cu_sel[b + 1] - cu_sel[b];
        if (n == 0) continue;
        // (factors are for 16 rows of the cache: contexts have to begin with one; and the bf16 kernel expects a token's row to exist)
        if (ctx_off[b] % kAlign || n > ctx_len[b]) return false;
        flops += 256.0 * shape->n_q_heads * (double)n * (double)ctx_len[b];
        bytes += 768.0 * shape->n_kv_heads * (double)ctx_len[b];
    }
    return flops * (1 / (cache->code == KVS_E4M3 ? 0.66e15 : 0.52e15) - 1 / 1.05e15) > bytes / 4.5e12 + 55e-6;
}

// *taken: whether the launch was made (it is not where the workspace is too small for the copy, or the bf16 kernel would not take it)
kvs_status launch_from_copy(const kvs_shape *shape, const kvs_cache8 *c, int32_t n_req, const int64_t *ctx_off, const int64_t *ctx_len, const int64_t *cu_sel,
                            const void *q_sel, const int32_t *sel_pos, float scale, void *out, float *lse_out, void *workspace, size_t workspace_bytes,
                            hipStream_t hs, bool *taken)
{
    CopyRanges cr = {};
    AttnBatch bd = {};
    int order[kAttnMaxReq];                // the requests that select tokens, by their first row
    int n_live = 0;
    for (int b = 0; b < n_req; ++b) {
        if (cu_sel[b + 1] == cu_sel[b]) continue;
        int j = n_live++;
        while (j > 0 && ctx_off[order[j - 1]] > ctx_off[b]) { order[j] = order[j - 1]; --j; }
        order[j] = b;
    }
    int64_t groups = 0, end = -1;          // of the copy so far; the last range's, in the cache, a multiple of 16
    auto close = [&] { if (cr.n > 0) groups += (end - cr.row[cr.n - 1]) / kAlign + 1; };   // (whole tiles of 32 keys have factors)
    for (int i = 0; i < n_live; ++i) {
        const int b = order[i];
        const int64_t to = (ctx_off[b] + ctx_len[b] + kAlign - 1) / kAlign * kAlign;
        if (cr.n == 0 || ctx_off[b] > end) {
            close();
            if (groups > 0x7fffff) return KVS_OK;
            cr.row[cr.n] = ctx_off[b];
            cr.begin[cr.n++] = (int32_t)groups;
            end = to;
        } else if (to > end) {
            end = to;
        }
        bd.ctx_off[b] = groups * kAlign + ctx_off[b] - cr.row[cr.n - 1];
        bd.ctx_len[b] = ctx_len[b];
    }
    close();
    if (groups > 0x7fffff) return KVS_OK;
    for (int b = cr.n; b <= kAttnMaxReq; ++b) cr.begin[b] = (int32_t)groups;
    for (int b = 0; b <= kAttnMaxReq; ++b) bd.cu_sel[b] = cu_sel[b < n_req ? b : n_req];
    bd.sel_begin = cu_sel[0];
    bd.n_req = n_req;
    const size_t need = copy_bytes(shape, groups);
    if (workspace_bytes < need + 256) return KVS_OK;
    const size_t left = (workspace_bytes - need) / 256 * 256;        // the bf16 kernel's, in front of the copy
    AttnSplitPlan plan;
    if (!attention_takes_large(shape, bd, left, &plan)) return KVS_OK;
    *taken = true;
    const int64_t rows = groups * kAlign;
    char *at = (char *)workspace + left;
    uint4 *k_copy = (uint4 *)at, *v_copy = (uint4 *)(at + rows * shape->n_kv_heads * 256);
    float4 *factors = (float4 *)(at + rows * shape->n_kv_heads * 512);
    const int64_t stride = groups + kCopyPad;
    const float scale_log2 = scale * 1.4426950408889634f;
    const dim3 grid((unsigned)groups), threads(kCopyThreads);
#define KVS_COPY(C) hipLaunchKernelGGL((copy8_kernel<C>), grid, threads, 0, hs, cr, shape->n_kv_heads, c->n_rows, __builtin_ctz((unsigned)c->block), \
                                       (const uint4 *)c->k, (const uint4 *)c->v, c->k_scale, c->v_scale, scale_log2, k_copy, v_copy, factors, stride)
    if (c->code == KVS_E4M3) KVS_COPY(KVS_E4M3); else KVS_COPY(KVS_INT8);
#undef KVS_COPY
    kvs_status st = check_launch("kvs_attention_kv8(copy)");
    if (st != KVS_OK) return st;
    st = launch_attention_mfma2(shape, bd, q_sel, sel_pos, k_copy, v_copy, scale, out, lse_out, left ? workspace : nullptr, left, plan, hs, {factors, stride});
    if (st != KVS_OK) return st;
    const int64_t n_sel = cu_sel[n_req] - cu_sel[0];
    hipLaunchKernelGGL(empty_rows_kernel, dim3((unsigned)((n_sel + kWaves - 1) / kWaves)), dim3(kThreads), 0, hs, n_sel, shape->n_q_heads, sel_pos + cu_sel[0],
                       (uint4 *)out + cu_sel[0] * shape->n_q_heads * 16, lse_out ? lse_out + cu_sel[0] * shape->n_q_heads : nullptr);
    return check_launch("kvs_attention_kv8(rows)");
}

template <int DTYPE, int CODE, int D, int PARTS>
kvs_status launch(const kvs_shape *shape, const kvs_cache8 *c, const Table &td, int64_t wgs, const void *q_sel, const int32_t *sel_pos, float scale,
                  void *out, float *lse_out, float *part_o, float4 *part_ml, hipStream_t hs)
{
    static DeviceOnce once;
    constexpr int lds = kWaves * 4 * kKeys * D;
    const kvs_status st = once_per_device(once, [&]() -> kvs_status {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attention8_kernel<DTYPE, CODE, D, PARTS>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        return e == hipSuccess ? KVS_OK : fail(KVS_EHIP, "kvs_attention_kv8: %s", hipGetErrorString(e));
    });
    if (st != KVS_OK) return st;
    hipLaunchKernelGGL((attention8_kernel<DTYPE, CODE, D, PARTS>), dim3((unsigned)wgs), dim3(kThreads), lds, hs, td, shape->n_q_heads, shape->n_kv_heads, c->n_rows,
                       __builtin_ctz((unsigned)c->block), (const uint8_t *)c->k, (const uint8_t *)c->v, c->k_scale, c->v_scale, q_sel, sel_pos,
                       scale * 1.4426950408889634f, out, lse_out, part_o, part_ml);
    return check_launch("kvs_attention_kv8");
}

} // namespace

size_t attention8_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t n_rows_total, int64_t n_sel_total)
{
    // a launch that is cut has at most kMaxCutWgs workgroups, of 32 rows each
    if (check_shape(shape) != KVS_OK || n_sel_total <= 0) return 256;
    int64_t pieces = tiles_of(n_rows_total) / kMinPieceTiles + 1;
    if (pieces > kMaxPieces) pieces = kMaxPieces;
    const int64_t most = (int64_t)kRows * kMaxCutWgs;
    int64_t slots = most;
    if (n_sel_total < most && n_sel_total * shape->n_q_heads < most) slots = n_sel_total * shape->n_q_heads * pieces < most ? n_sel_total * shape->n_q_heads * pieces : most;
    size_t bytes = ((size_t)slots * slot_bytes(shape->head_dim) + 255) / 256 * 256;
    if (shape->dtype == KVS_BF16 && shape->head_dim == 128 && n_sel_total >= kCopyMinRows / shape->n_q_heads) {
        const size_t copy = (copy_bytes(shape, copy_groups(batch, n_rows_total)) + attention_workspace_bytes(shape, batch, n_rows_total, n_sel_total) + 511) / 256 * 256;
        if (copy > bytes) bytes = copy;
    }
    return bytes;
}

} // namespace kvs

extern "C" kvs_status kvs_attention_kv8(const kvs_shape *shape, const kvs_cache8 *cache, int32_t batch,
                                        const int64_t *ctx_off, const int64_t *ctx_len, const int64_t *cu_sel,
                                        const void *q_sel, const int32_t *sel_pos, float scale,
                                        void *out, float *lse_out, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace kvs;
    const char *me = "kvs_attention_kv8";
    kvs_status st = check_shape(shape);
    if (st != KVS_OK || (st = check_cache8(me, shape, cache)) != KVS_OK) return st;
    if (batch < 0) return fail(KVS_EINVAL, "%s: batch < 0", me);
    if (!isfinite(scale)) return fail(KVS_EINVAL, "%s: the scale is not finite", me);
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(KVS_EINVAL, "%s: workspace must be 256-byte aligned", me);
    if (!workspace) workspace_bytes = 0;
    if (batch == 0) return KVS_OK;
    if (!ctx_off || !ctx_len || !cu_sel) return fail(KVS_EINVAL, "%s: ctx_off/ctx_len/cu_sel is NULL", me);
    if (cu_sel[0] != 0) return fail(KVS_EINVAL, "%s: cu_sel[0] must be 0", me);
    const int grp = shape->n_q_heads / shape->n_kv_heads;
    for (int32_t b = 0; b < batch; ++b) {
        if (ctx_off[b] < 0 || ctx_len[b] < 0 || ctx_off[b] > cache->n_rows - ctx_len[b])
            return fail(KVS_EINVAL, "%s: request %d's rows %lld .. +%lld lie outside a cache of %lld", me, b, (long long)ctx_off[b], (long long)ctx_len[b], (long long)cache->n_rows);
        if (ctx_len[b] > 0x7fffff00LL) return fail(KVS_EINVAL, "%s: context of request %d too long", me, b);
        if (cu_sel[b + 1] < cu_sel[b]) return fail(KVS_EINVAL, "%s: cu_sel decreases at request %d", me, b);
        if ((cu_sel[b + 1] - cu_sel[b]) > 0x7fffff00LL / shape->n_q_heads) return fail(KVS_EINVAL, "%s: request %d selects too many tokens", me, b);
    }
    if (cu_sel[batch] == 0) return KVS_OK;
    if (!q_sel || !sel_pos || !out) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    if (!aligned16(q_sel) || !aligned16(out)) return fail(KVS_EINVAL, "%s: Q/out pointers must be 16-byte aligned", me);
    hipStream_t hs = (hipStream_t)stream;
    for (int32_t b0 = 0; b0 < batch; b0 += kAttnMaxReq) {
        const int nr = (batch - b0) < kAttnMaxReq ? (batch - b0) : kAttnMaxReq;
        const int64_t n_sel = cu_sel[b0 + nr] - cu_sel[b0];
        if (n_sel == 0) continue;
        if (n_sel > 0x7fffff00LL / shape->n_q_heads) return fail(KVS_EINVAL, "%s: %lld selected tokens in one launch", me, (long long)n_sel);
        if (bf16_copy_pays(shape, cache, nr, ctx_off + b0, ctx_len + b0, cu_sel + b0, scale)) {
            bool taken = false;
            st = launch_from_copy(shape, cache, nr, ctx_off + b0, ctx_len + b0, cu_sel + b0, q_sel, sel_pos, scale, out, lse_out, workspace, workspace_bytes, hs, &taken);
            if (st != KVS_OK) return st;
            if (taken) continue;
        }
        const Plan plan = plan_pieces(shape, nr, ctx_len + b0, cu_sel + b0, workspace_bytes);
        Table td = {};
        td.n_req = nr;
        td.sel0 = cu_sel[b0];
        td.piece_tiles = plan.piece_tiles ? (int32_t)plan.piece_tiles : 0x7fffffff;
        int64_t units = 0, slot = 0, most = 0;
        int32_t most_pieces = 1;
        for (int i = 0; i < kAttnMaxReq; ++i) {
            td.unit_begin[i] = (int32_t)units;
            td.sel_begin[i] = i < nr ? (int32_t)(cu_sel[b0 + i] - cu_sel[b0]) : (int32_t)n_sel;
            if (i >= nr) continue;
            const int64_t n = cu_sel[b0 + i + 1] - cu_sel[b0 + i];
            const int64_t p = n && plan.piece_tiles ? (tiles_of(ctx_len[b0 + i]) + plan.piece_tiles - 1) / plan.piece_tiles : 1;
            td.ctx_off[i] = ctx_off[b0 + i];
            td.slot_begin[i] = (int32_t)slot;
            td.ctx_len[i] = (int32_t)ctx_len[b0 + i];
            td.pieces[i] = (int32_t)(p > 1 ? p : 1);
            if (p > 1) slot += n * shape->n_q_heads * p;
            const int64_t own = blocks_of(n, grp) * td.pieces[i];
            units += own;
            if (own > most) most = own;
            if (td.pieces[i] > most_pieces) most_pieces = td.pieces[i];
            if (units * shape->n_kv_heads > 0x7fffffff / kThreads) return fail(KVS_EINVAL, "%s: too many rows in one launch", me);
        }
        td.unit_begin[kAttnMaxReq] = (int32_t)units;
        // In a launch of few rounds all requests' longest units begin (8 contexts of 4000 to 8000 under 100 rows each: 105 us one
        // request after the other, 88 so), unless that leaves many workgroups without a unit.  In longer ones a request's
        // row blocks stay together, which share its keys in L2 (32 contexts under 160 rows: 850 us, 1020 interleaved).
        td.interleaved = nr > 1 && units * shape->n_kv_heads <= kMaxCutWgs && most * nr <= units + units / 4;
        if (td.interleaved) units = most * nr;
        td.sel_begin[kAttnMaxReq] = (int32_t)n_sel;
        float4 *ml = reinterpret_cast<float4 *>(workspace);
        float *po = reinterpret_cast<float *>(ml + plan.slots);
        const int64_t wgs = units * shape->n_kv_heads, items = n_sel * shape->n_q_heads;
        // Weights of launches that the caches' bytes bound enter the second product as two bf16, which costs up to 4% there (131072
        // keys 35.3 -> 36.7 us, 64 of 4096 to 16384 the same); with several blocks a request it would be 8 to 11%.
        bool one_block = true;
        for (int i = 0; i < nr; ++i) one_block = one_block && blocks_of(cu_sel[b0 + i + 1] - cu_sel[b0 + i], grp) <= 1;
        const bool e4m3 = cache->code == KVS_E4M3, wide = shape->head_dim == 128, bf16 = shape->dtype == KVS_BF16;
#define KVS_A8(DT, C, DD, PP) launch<DT, C, DD, PP>(shape, cache, td, wgs, q_sel, sel_pos, scale, out, lse_out, po, ml, hs)
#define KVS_A8_OF(DT, PP) (e4m3 ? (wide ? KVS_A8(DT, KVS_E4M3, 128, PP) : KVS_A8(DT, KVS_E4M3, 64, PP)) : (wide ? KVS_A8(DT, KVS_INT8, 128, PP) : KVS_A8(DT, KVS_INT8, 64, PP)))
        if (!bf16) st = KVS_A8_OF(KVS_F32, 3);
        else if (one_block) st = KVS_A8_OF(KVS_BF16, 2);
        else st = KVS_A8_OF(KVS_BF16, 1);
#undef KVS_A8_OF
#undef KVS_A8
        if (st != KVS_OK) return st;
        if (!plan.piece_tiles) continue;
        const dim3 threads(kThreads);
        const int per_wg = kThreads / (shape->head_dim / 4);
#define KVS_M8(DT, DD)                                                                                                                                    \
    do {                                                                                                                                                  \
        if (most_pieces <= kFewPieces)                                                                                                                    \
            hipLaunchKernelGGL((merge8_rows_kernel<DT, DD>), dim3((unsigned)((items + per_wg - 1) / per_wg)), threads, 0, hs, td, (int)items,             \
                               shape->n_q_heads, po, ml, out, lse_out);                                                                                   \
        else hipLaunchKernelGGL((merge8_kernel<DT, DD>), dim3((unsigned)items, DD / 32), threads, 0, hs, td, shape->n_q_heads, po, ml, out, lse_out);    \
    } while (0)
        if (bf16) { if (wide) KVS_M8(KVS_BF16, 128); else KVS_M8(KVS_BF16, 64); }
        else { if (wide) KVS_M8(KVS_F32, 128); else KVS_M8(KVS_F32, 64); }
#undef KVS_M8
        if ((st = check_launch("kvs_attention_kv8")) != KVS_OK) return st;
    }
    return KVS_OK;
}
