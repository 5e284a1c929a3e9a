// kvs_attention_paged: attention of new or selected tokens over a cache in pages, with an optional sliding window beside a few first
// tokens that stay visible.
//
// Mathematics.  out = sum_i p_i v_i / sum_i p_i with p_i = exp(scale q . k_i - max) over the keys that the row sees: one pass
// over the keys with a running maximum and sum.
//
// Tiles.  A wave takes 32 rows (the query heads of one KV head flattened with the tokens) against tiles of 32 keys, S^T = K Q^T and
// O^T += V^T P^T, so that P stays in registers as the operand of the second product.  A tile is two runs of 16 rows, each in
// one page; the wave's next 32 tiles' places are kept in its lanes, two a tile, and read from them without a trip to memory.
// Under a window a row block's tiles are those of the first tokens and those from its lowest row's window on; the others are
// not counted, loaded or computed.
//
// The four waves of a workgroup take the same 32 rows and every fourth tile, each with an LDS slot for K and one for V that its
// loads go to directly (global to LDS, 16 bytes a lane, no registers), without a barrier: K of the next tile is asked for once
// this tile's has been read, V likewise, so that a tile's worth of loads is under way all the time, and two workgroups share a CU (fp32 at
// 128 channels: one, whose slots take 128 KB).
// At the end the waves meet in LDS.  Launches of too few workgroups cut the keys into pieces, which a second kernel merges.
//
// Measured (bf16, 128 channels, one token a request, 28 or 32 query heads).  Memory bounds the long ones: 131072 keys of 4 KV heads, 268 MB, 44.5 us and
// 4.8 for the merge, 6.0 TB/s; 64 contexts of 4096 to 16384 of 8 KV heads, 2.6 GB, 435 us, 6.0 TB/s.  The short ones are a chain of trips: launch and
// length 2, Q and the first keys, the meeting, 6.0 us up to 128 keys, and 1.0 more for every further tile of a wave, since only one is under way: 601
// keys 10.7.  (Eight waves a workgroup instead: 601 keys 10.0, but 1000 11.4 for 10.7 and 128 7.1 for 6.2.)
//
// fp32 goes through the fp32 matrix instruction, whose operands need no other order than that of memory.
#include "attention_paged.h"

#include <math.h>

namespace kvs {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kRows = 32;              // rows of a block
constexpr int kKeys = 32;              // keys of a tile
constexpr float kSlack = 8.f;          // powers of two that a score may lie above its reference
constexpr int kMaxPieces = kPagedMaxPieces;
constexpr int kPlaces = 512;           // workgroups that the chip holds at once

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

__device__ __forceinline__ float max_of_halves(float x)      // of lanes i and i + 32
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// PARTS: bf16 numbers that a weight enters the second product as: one, or two that hold 16 of its bits (fp32: the weights are what they are).  One is
// off by up to 2^-8 (rounding the output to bf16 is off by as much); a second one would be half as many products again, which bound launches of many rows,
// and is nearly free where memory does.
// So two go with few rows a request: K and V are then read once, and their loads say so (64 contexts of 4096 to 16384 487 -> 443 us, 131072
// keys 59 -> 53; where several blocks share the keys through L2, 24 tokens over each of 8 contexts, 83 -> 100).
// AGAIN: the rows of row tiles of 256 whose kernel asks for it (`odd`, a word a workgroup of its), eight blocks each.
template <int DTYPE, int D, int PARTS, bool AGAIN>
__global__ __launch_bounds__(kThreads, DTYPE == KVS_F32 && D == 128 ? 1 : 2) void attention_paged_kernel(
    const Paged pg, int n_q_heads, int n_kv_heads, int units, int pieces, int least_tiles, const int32_t *__restrict__ odd,
    const char *__restrict__ k_pool, const char *__restrict__ v_pool, const void *__restrict__ q_new, float scale_log2,
    void *__restrict__ out, float *__restrict__ lse_out, float *__restrict__ part_o, float4 *__restrict__ part_ml)
{
    constexpr bool F32 = DTYPE == KVS_F32;
    constexpr int ES = F32 ? 4 : 2;
    constexpr int NDB = D / 32;
    constexpr int ROW_B = D * ES;
    constexpr int CPR = ROW_B / 16;                          // 16-byte chunks of a row
    constexpr int RPL = kWave / CPR;                         // rows a load moves
    constexpr int NH = kGranule / RPL;                       // loads of half a tile
    constexpr int NL = 2 * NH;
    constexpr int TILE_B = kKeys * ROW_B;
    constexpr int WAVE_B = 2 * TILE_B;                       // a slot for K, one for V
    constexpr int MEET_B = kRows * D * 4;                    // the wave's sums at the end
    static_assert(MEET_B <= WAVE_B, "the sums take the slots' place");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float4 ml_s[kWaves][kRows];
    __shared__ int odd_s;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hf = lane >> 5, ln = lane & 31;

    const PagedPlace at = place_of(blockIdx.x, units, AGAIN ? 1 : pieces, n_kv_heads);
    const int g = __builtin_amdgcn_readfirstlane(at.g), piece = __builtin_amdgcn_readfirstlane(at.piece), unit = __builtin_amdgcn_readfirstlane(at.unit);
    const int grp = n_q_heads / n_kv_heads;
    Block found;
    if constexpr (AGAIN) {
        int any = 0;
        for (int p = 0; p < pieces; ++p) any |= odd[(p * units + unit) * n_kv_heads + g];
        if (!any || !find_block<kPagedLargeRows>(pg, grp, units - 1 - unit, found)) return;
        pieces = 1;
    } else {
        if (!find_block<kRows>(pg, grp, unit, found)) return;
    }
    const int b = __builtin_amdgcn_readfirstlane(found.b), blk = __builtin_amdgcn_readfirstlane(found.blk), tok0 = __builtin_amdgcn_readfirstlane(found.tok0);
    const int n_tok = __builtin_amdgcn_readfirstlane(found.n_tok), len = __builtin_amdgcn_readfirstlane(found.len), end = __builtin_amdgcn_readfirstlane(found.end);
    const int rows = n_tok * grp;

    // Without a window the first piece's tiles do not depend on the length, and their places are asked for beside it.
    const bool known = !AGAIN && !pg.window && piece == 0;
    const int early = known ? granule_of(pg, b, 2 * (wave + kWaves * (lane >> 1)) + (lane & 1)) : -1;
    auto block_from = [&](const int row0) __attribute__((always_inline)) {
    // ---- this lane's row (both half-waves hold the same 32) ------------------------------------------------
    const int rq = min(max(row0 + ln, 0), rows - 1);
    const int t_own = rq / grp, hh = rq - t_own * grp;
    const int pos = position_of(pg, tok0, n_tok, t_own, len, end);
    int pmin = pos, pmax = pos, plow = pos < 0 ? 0x7fffffff : pos;        // plow: of those that see anything
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        pmin = min(pmin, __shfl_xor(pmin, o));
        pmax = max(pmax, __shfl_xor(pmax, o));
        plow = min(plow, __shfl_xor(plow, o));
    }
    pmin = __builtin_amdgcn_readfirstlane(pmin);
    pmax = __builtin_amdgcn_readfirstlane(pmax);
    plow = __builtin_amdgcn_readfirstlane(plow);
    const int window = pg.window, n_first = window ? pg.n_first : 0;
    const int below = window ? pos - window : -1;            // keys up to here are seen only if they are first ones

    // ---- the block's tiles: `head` tiles from 0 on, then those from `low` on ------------------------------
    const int low = window && pmax >= 0 ? max(plow - window + 1, 0) / kKeys : 0;
    const int head = min(low, (int)(((int64_t)n_first + kKeys - 1) / kKeys));
    const int total = pmax < 0 ? 0 : head + pmax / kKeys + 1 - low;
    // equal pieces of what there is, none below least_tiles
    const int piece_tiles = max(((total + pieces - 1) / pieces + kWaves - 1) / kWaves * kWaves, least_tiles);
    const int t_lo = (int)min((int64_t)piece * piece_tiles, (int64_t)total), t_hi = (int)min((int64_t)t_lo + piece_tiles, (int64_t)total);
    const int mine = max(0, (t_hi - t_lo - wave + kWaves - 1) / kWaves);
    auto tile_of = [&](int i) { const int t = t_lo + wave + kWaves * i; return t < head ? t : t - head + low; };

    if (t_lo >= t_hi && pieces > 1) {                        // nothing for the merge
        if (wave == 0 && hf == 0 && row0 + ln < rows)
            part_ml[((int64_t)(tok0 + t_own) * n_q_heads + g * grp + hh) * pieces + piece] = make_float4(kLowest, 0.f, 0.f, 0.f);
        return;
    }

    // places of tiles i0 .. i0 + 31 (two a tile); -1 where the table names no page
    int place = -1;
    auto look_up = [&](int i0) {
        const int i = i0 + (lane >> 1);
        place = i < mine ? granule_of(pg, b, 2 * tile_of(i) + (lane & 1)) : -1;
    };
    if (!known) look_up(0);
    else place = (lane >> 1) < mine ? early : -1;

    // ---- Q as the B operand; a negative scale's sign goes into it, so that the largest score is the largest product's ----
    const bool negative = scale_log2 < 0.f;
    const float scale_abs = fabsf(scale_log2);
    u32x4_t qreg[D / (F32 ? 8 : 16)];
    {
        const char *at = (const char *)q_new + (((int64_t)(tok0 + t_own) * n_q_heads + g * grp + hh) * D) * ES;
#pragma unroll
        for (int ks = 0; ks < D / (F32 ? 8 : 16); ++ks) {
            u32x4_t w = *reinterpret_cast<const u32x4_t *>(at + 32 * ks + 16 * hf);
            if constexpr (F32) w ^= (negative ? 0x80000000u : 0u);
            else w ^= (negative ? 0x80008000u : 0u);
            qreg[ks] = w;
        }
    }

    // ---- staging ------------------------------------------------------------------------------------------------
    // A load moves RPL rows, 16 bytes a lane, to consecutive LDS.  Chunk c of row r lies at c ^ swz(r): K's for lanes that read one
    // chunk of many rows, V's for the transposing reads of four rows.
    char *const my_lds = lds + wave * WAVE_B;
    char *const kt = my_lds, *const vt = my_lds + TILE_B;
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)my_lds);
    const uint32_t row_bytes = (uint32_t)n_kv_heads * ROW_B;
    auto k_swz = [](int r) { return CPR >= 16 ? (r & 15) : (r & 7); };
    auto v_swz = [](int r) { return F32 ? (CPR >= 16 ? (r & 15) : (r & 7)) : CPR >= 16 ? 2 * (r & 7) : 2 * (r & 3); };
    const int st_row = lane / CPR, st_at = lane % CPR;
    uint32_t k_off[NH], v_off[NH];
#pragma unroll
    for (int j = 0; j < NH; ++j) {
        const int r = j * RPL + st_row;
        k_off[j] = (uint32_t)r * row_bytes + (uint32_t)(st_at ^ k_swz(r)) * 16u;
        v_off[j] = (uint32_t)r * row_bytes + (uint32_t)(st_at ^ v_swz(r)) * 16u;
    }
    // Written by hand: issued through the compiler's builtin, every later LDS read would wait for all loads in flight.  M0 holds
    // the LDS address of lane 0; the nop is the wait state that a write to M0 needs before such a load.
    auto load_1k = [&](uint32_t dst, uint32_t off, const char *base) {
        if constexpr (PARTS == 2) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(dst), "v"(off), "s"(base) : "memory");
        else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst), "v"(off), "s"(base) : "memory");
    };
    const uint64_t granule_bytes = (uint64_t)row_bytes * kGranule;
    auto stage = [&](int i, const char *pool, const uint32_t (&off)[NH], uint32_t dst) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = max(__builtin_amdgcn_readlane(place, 2 * (i & 31) + h), 0);       // (no page: any rows, masked below)
            const char *base = pool + (uint64_t)(uint32_t)at * granule_bytes + (uint32_t)g * ROW_B;
#pragma unroll
            for (int j = 0; j < NH; ++j) load_1k(dst + (h * NH + j) * 1024, off[j], base);
        }
    };
    auto stage_k = [&](int i) { stage(i, k_pool, k_off, lds_base); };
    auto stage_v = [&](int i) { stage(i, v_pool, v_off, lds_base + TILE_B); };

    // ---- running state ------------------------------------------------------------------------------------------
    floatx16 o_acc[NDB];
    float m_run, l_run, l_rnd;
    // entry r of the score accumulator is key `entry(r) + (F32 ? 4 : 8) hf` of the tile: K rows are fed to the bf16 instruction with bits 2
    // and 3 swapped, so that a lane's weights are 8 consecutive keys twice
    const int krow = F32 ? ln : (ln & ~12) | ((ln & 4) << 1) | ((ln & 8) >> 1);
    constexpr int HALF = F32 ? 4 : 8;
    auto entry = [](int r) { return F32 ? 8 * (r >> 2) + (r & 3) : 16 * (r >> 3) + (r & 7); };
    const int tr_s = lane & 15, tr_g = lane >> 4;                        // (see read_v)
    const int tr_key = 8 * (tr_g >> 1) + (tr_s >> 2), tr_c = 2 * (tr_g & 1) + ((tr_s & 3) >> 1);
    auto read_v = [&](int a, int db) -> u32x4_t {
        // The A operand of the second product: channel 32 db + ln, 8 consecutive keys, out of two transposing reads: in each
        // group of 16 lanes, lane s points at 4 channels of key s / 4 and lane i receives channel i of the four keys.
        typedef short v4i16 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
        u32x4_t r;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int key = 16 * a + tr_key + 4 * u;
            const char *at = vt + key * ROW_B + ((4 * db + tr_c) ^ v_swz(key)) * 16 + 8 * (tr_s & 1);
            const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(at)));
            r[2 * u] = w.x;
            r[2 * u + 1] = w.y;
        }
        return r;
    };
    auto v_element = [&](int key, int c) -> float {
        const char *at = vt + key * ROW_B + ((c * ES / 16) ^ v_swz(key)) * 16 + (c * ES) % 16;
        if constexpr (F32) return *reinterpret_cast<const float *>(at);
        else return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(at) << 16);
    };

    // A weight of 0 does not hide a V that is infinite or NaN.  Rows behind the context, and of no page, are cleared in LDS.  Others, in a
    // tile that some row does not see all of, are found out at the end: an output that is no number makes the workgroup sweep once
    // more, carefully, where such keys are multiplied with the weights of the rows that see them, and no others.
    for (int careful = 0; careful < 2; ++careful) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o_acc[db][r] = 0.f;
        m_run = kLowest;           // reference of the weights: a former maximum of the scores times log2 e, the same in both half-waves
        l_run = l_rnd = 0.f;       // this half-wave's share of the sum of weights; the same of the weights as the second product sees them
        if (careful) look_up(0);
        if (mine > 0) { stage_k(0); stage_v(0); }
        for (int i = 0; i < mine; ++i) {
            const int x0 = tile_of(i) * kKeys;
            const bool none[2] = {__builtin_amdgcn_readlane(place, 2 * (i & 31)) < 0, __builtin_amdgcn_readlane(place, 2 * (i & 31) + 1) < 0};
            const bool more = i + 1 < mine;
            asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NL) : "memory");           // K has landed, V may still be on its way
            if (more && ((i + 1) & 31) == 0) look_up(i + 1);

            floatx16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < CPR / 2; ++c) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t *>(kt + krow * ROW_B + ((2 * c + hf) ^ k_swz(krow)) * 16);
                if constexpr (F32) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[u]), __uint_as_float(qreg[c][u]), s, 0, 0, 0);
                } else {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w), as_bf16x8(qreg[c]), s, 0, 0, 0);
                }
            }
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");               // what lay in the slot has been read
                stage_k(i + 1);
            }
            const bool masked = x0 + kKeys - 1 > pmin || none[0] || none[1] || (window && x0 <= pmax - window && x0 + kKeys > n_first);
            float f = scale_abs;
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = x0 + entry(r) + HALF * hf;
                    const bool seen = key <= pos && (key > below || key < n_first) && !none[r >> 3];
                    s[r] = seen ? s[r] * f : -INFINITY;
                }
                f = 1.f;
            }
            float mx = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
            mx = max_of_halves(mx) * f;
            // The reference that weights are relative to moves only once a score is kSlack above it (in powers of two): weights of up
            // to 2^kSlack lose nothing, and sums are seldom scaled behind a row's first tiles.
            if (__builtin_amdgcn_ballot_w64(mx > m_run + kSlack) != 0) {
                const float m_new = fmaxf(m_run, mx), corr = __builtin_amdgcn_exp2f(m_run - m_new);
                m_run = m_new;
                l_run *= corr;
                l_rnd *= corr;
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o_acc[db][r] *= corr;
            }
            float y[16], psum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                y[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], f, -m_run));
                psum += y[r];
            }
            l_run += psum;
            u32x4_t pop[F32 ? 1 : 2][F32 ? 1 : PARTS];
            if constexpr (!F32) {
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float u = y[8 * a + 2 * j], v = y[8 * a + 2 * j + 1];
                        const uint32_t w = pack2(u, v);
                        pop[a][0][j] = w;
                        if constexpr (PARTS == 2) pop[a][1][j] = pack2(u - bf16_lo(w), v - bf16_hi(w));
                        // One part: the normaliser is made of the rounded weights.  Numerator and denominator then carry the same rounding, and a
                        // row that one key dominates returns that key's V to within the output's own rounding.
                        else l_rnd = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), l_rnd, false);
                    }
            }

            if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NL) : "memory");      // V has landed, the next K may still be on its way
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (x0 + kKeys > len || none[0] || none[1]) {
#pragma unroll
                for (int e = 0; e < TILE_B / 1024; ++e) {
                    const int r = (e * kWave + lane) / CPR;
                    if (x0 + r >= len || none[r >> 4]) reinterpret_cast<u32x4_t *>(vt)[e * kWave + lane] = u32x4_t{0u, 0u, 0u, 0u};
                }
            }
            if (careful && masked) {
                // Next K is on its way into its slot, so the weights change hands through the registers, key by key.
                for (int key = 0; key < kKeys; ++key) {
                    bool odd = false;
                    for (int c = lane; c < D; c += kWave) odd = odd || !(fabsf(v_element(key, c)) < INFINITY);
                    if (__builtin_amdgcn_ballot_w64(odd) == 0) continue;
                    const int from = (key / HALF) & 1;                    // the half-wave that holds the key's weights, and their place in it
                    const int at = F32 ? 4 * (key >> 3) + (key & 3) : 8 * (key >> 4) + (key & 7);
                    float p = y[0];
#pragma unroll
                    for (int r = 1; r < 16; ++r) p = r == at ? y[r] : p;
                    p = __shfl(p, ln + 32 * from);
                    const int k_at = x0 + key;
                    const bool seen = k_at <= pos && (k_at > below || k_at < n_first) && !none[key >> 4];
                    if (seen) {
                        p = fmaxf(p, 1e-37f);
#pragma unroll
                        for (int db = 0; db < NDB; ++db)
#pragma unroll
                            for (int r = 0; r < 16; ++r) o_acc[db][r] += p * v_element(key, 32 * db + 8 * (r >> 2) + 4 * hf + (r & 3));
                    }
                    if (lane < CPR) *reinterpret_cast<u32x4_t *>(vt + key * ROW_B + lane * 16) = u32x4_t{0u, 0u, 0u, 0u};
                }
            }
            if constexpr (F32) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
                        o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v_element(entry(r) + HALF * hf, 32 * db + ln), y[r], o_acc[db], 0, 0, 0);
            } else {
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int db = 0; db < NDB; ++db) {
                        const u32x4_t va = read_v(a, db);
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(va), as_bf16x8(pop[a][p]), o_acc[db], 0, 0, 0);
                    }
            }
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                stage_v(i + 1);
            }
        }

        // ---- the waves meet ----------------------------------------------------------------------------------------
        {
            const float l = l_run + __shfl_xor(l_run, 32), lr = l_rnd + __shfl_xor(l_rnd, 32);
            if (hf == 0) ml_s[wave][ln] = make_float4(m_run, l, !F32 && PARTS == 1 ? lr : l, 0.f);
            if (tid == 0) odd_s = 0;
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
        const int row_q = row0 + row;
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
                const float4 x = *reinterpret_cast<const float4 *>(from + 4 * ((CPT / 4 * part + k) ^ (row & (D / 4 - 1))));
                o[4 * k] += x.x; o[4 * k + 1] += x.y; o[4 * k + 2] += x.z; o[4 * k + 3] += x.w;
            }
        }
        if (!careful) {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < CPT; ++c) sum += o[c] * 0.f;                  // 0, or NaN
            if (!(sum == 0.f)) odd_s = 1;
            __syncthreads();
            if (odd_s) { __syncthreads(); continue; }
        }
        if (row_q >= rows || row_q < 0) return;
        const int t2 = row_q / grp;
        const int64_t at = (int64_t)(tok0 + t2) * n_q_heads + g * grp + (row_q - t2 * grp);
        if (pieces > 1) {
            const int64_t slot = at * pieces + piece;
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
        if constexpr (!F32) {
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
        return;
    }
    };
    // (row tiles of 256 end with their request's rows)
    if constexpr (AGAIN) {
        const int first = blk * kPagedLargeRows - ((rows + kPagedLargeRows - 1) / kPagedLargeRows * kPagedLargeRows - rows);
        for (int r = 0; r < kPagedLargeRows; r += kRows) {
            if (first + r + kRows <= 0) continue;
            block_from(first + r);
            __syncthreads();
        }
    } else {
        block_from(blk * kRows);
    }
}

// out = sum_p w_p O_p / sum_p w_p l_p with w_p = 2^(m_p - max m).  A workgroup takes 32 channels of one row: its threads make the
// pieces' weights once, into LDS, then groups of 8 threads take every 32nd piece, four channels a thread, and meet by shuffles and in LDS.
template <int DTYPE, int D>
__global__ __launch_bounds__(kThreads) void merge_paged_kernel(const Paged pg, int n_q_heads, int pieces, const float *__restrict__ part_o,
                                                               const float4 *__restrict__ part_ml, void *__restrict__ out, float *__restrict__ lse_out)
{
    constexpr int kLanes = 8, kGroups = kThreads / kLanes;
    __shared__ float weight[kMaxPieces];
    __shared__ float meet[3][kWaves];
    __shared__ float4 sum_s[kWaves][kLanes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t item = blockIdx.x;
    if (pg.cu_new) {                                         // tokens of no request stay as they are
        const int token = (int)(item / n_q_heads);
        if (token < pg.cu_new[0] || token >= pg.cu_new[pg.batch]) return;
    }
    const int64_t slot = item * pieces;
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
        if (f == -1.f) continue;
        const float4 y = from[(int64_t)p * (D / 4)];
        o.x += f * y.x; o.y += f * y.y; o.z += f * y.z; o.w += f * y.w;
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
    const float inv = 1.f / lr;
    if (l != 0.f) { o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv; }
    else o = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (DTYPE == KVS_BF16) *reinterpret_cast<uint2 *>((uint16_t *)out + item * D + 4 * c) = make_uint2(pack2(o.x, o.y), pack2(o.z, o.w));
    else *reinterpret_cast<float4 *>((float *)out + item * D + 4 * c) = o;
    if (lse_out && c == 0) lse_out[item] = l != 0.f ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// The same with D / 4 threads a row, four channels a thread, and MOST pieces asked for at once.  (By the kernel above, 12800 rows of two
// pieces took 60 us: a workgroup for 32 channels of a row each.)
template <int DTYPE, int D, int MOST>
__global__ __launch_bounds__(kThreads) void merge_paged_rows_kernel(const Paged pg, int64_t n_items, int n_q_heads, int pieces, const float *__restrict__ part_o,
                                                                    const float4 *__restrict__ part_ml, void *__restrict__ out, float *__restrict__ lse_out)
{
    constexpr int kLanes = D / 4;
    const int c = threadIdx.x % kLanes;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    if (item >= n_items) return;
    if (pg.cu_new) {                                         // tokens of no request stay as they are
        const int token = (int)(item / n_q_heads);
        if (token < pg.cu_new[0] || token >= pg.cu_new[pg.batch]) return;
    }
    const int64_t slot = item * pieces;
    const float4 *from = reinterpret_cast<const float4 *>(part_o + slot * D) + c;
    float top = kLowest, l = 0.f, lr = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < pieces; p0 += MOST) {
        float4 x[MOST], y[MOST];
        float to = top;
#pragma unroll
        for (int p = 0; p < MOST; ++p) {
            x[p] = p0 + p < pieces ? part_ml[slot + p0 + p] : make_float4(kLowest, 0.f, 0.f, 0.f);
            y[p] = p0 + p < pieces ? from[(int64_t)(p0 + p) * kLanes] : make_float4(0.f, 0.f, 0.f, 0.f);
            to = fmaxf(to, x[p].x);
        }
        const float down = __builtin_amdgcn_exp2f(top - to);
        top = to;
        l *= down; lr *= down;
        o.x *= down; o.y *= down; o.z *= down; o.w *= down;
#pragma unroll
        for (int p = 0; p < MOST; ++p) {
            const float f = __builtin_amdgcn_exp2f(x[p].x - top);
            l += x[p].y * f;
            lr += x[p].z * f;
            if (x[p].y != 0.f) { o.x += f * y[p].x; o.y += f * y[p].y; o.z += f * y[p].z; o.w += f * y[p].w; }   // (a piece without keys has left no sums)
        }
    }
    const float inv = 1.f / lr;
    if (l != 0.f) { o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv; }
    else o = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (DTYPE == KVS_BF16) *reinterpret_cast<uint2 *>((uint16_t *)out + item * D + 4 * c) = make_uint2(pack2(o.x, o.y), pack2(o.z, o.w));
    else *reinterpret_cast<float4 *>((float *)out + item * D + 4 * c) = o;
    if (lse_out && c == 0) lse_out[item] = l != 0.f ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// Tiles that a block of rows may need at most.
int64_t most_tiles(const Paged &pg, int grp)
{
    int64_t keys = pg.max_ctx;
    if (pg.window && !pg.sel_pos) {                          // consecutive tokens: the window, and what 32 rows lie apart
        const int64_t some = (int64_t)pg.window + kRows / (grp < kRows ? grp : kRows) + 2 * kKeys + pg.n_first + kKeys;
        if (some < keys) keys = some;
    }
    return (keys + kKeys - 1) / kKeys + 1;
}

// How many pieces the keys are cut into, and about how long that takes.  The contexts' lengths are on the device, where every block of rows
// takes equal pieces of what it sees; the host knows how long a context can be.
struct Plan { int32_t pieces; double us; };
constexpr int kLeastTiles = kWaves;    // of a piece: one for each wave
constexpr int64_t kMostCutWgs = 4 * kPlaces;

// In microseconds, as measured: a step of four tiles, one a wave, takes 1.0, 1.5 beside a second workgroup on the compute unit, and workgroups
// beyond 512 wait for the first (fp32 at 128 channels has 256 places and is planned the same; 8192 keys of 8 heads 26 us, 256 tokens of 32 heads over
// 4096 162); the cache comes at 5.1 TB/s, and the two hide each other less the closer they are; where reading bounds the call
// or there are rounds, contexts of a batch that are longer than others hold the end up by a third of a piece, and the average one is shorter
// than the longest; 6 for the launch and a workgroup's beginning and end, 4 for a merge's.  Over 39 calls of 1 to 6000 tokens and 500 to 60000
// keys the kernel and number of pieces that this takes are within 10 % of the best there is in 35, within 22 % in all.
Plan plan_pieces(const kvs_shape *shape, const Paged &pg, const PagedCall &call, size_t workspace_bytes)
{
    const int64_t wgs = (int64_t)pg.batch * call.row_blocks * shape->n_kv_heads, most = most_tiles(pg, call.grp);
    const int64_t slots = (int64_t)(workspace_bytes / paged_slot_bytes(shape->head_dim)) / call.items;
    const double several = pg.batch > 1 ? 1.0 : 0.0;
    const double tile_bytes = 2.0 * kKeys * shape->head_dim * (shape->dtype == KVS_F32 ? 4 : 2);
    const double step = shape->dtype == KVS_F32 ? 2.5 : 1.0;              // (fp32's matrix instructions)
    const double reading = (double)pg.batch * shape->n_kv_heads * (double)most * tile_bytes * (1.0 - 0.25 * several) / 5.1e6;
    const int64_t even = shape->n_kv_heads % 8 == 0 ? 1 : shape->n_kv_heads % 4 == 0 ? 2 : shape->n_kv_heads % 2 == 0 ? 4 : 8;
    Plan best = {1, 1e30};
    auto consider = [&](int64_t p) {
        const int64_t n = p >= even ? (p + even - 1) / even * even : p;  // (see place_of)
        if (n > 1 && (n > slots || n > kMaxPieces || wgs * n > kMostCutWgs || (n - 1) * kLeastTiles >= most)) return false;
        const double steps = (double)((most + kWaves * n - 1) / (kWaves * n)), a_unit = (double)(wgs * n) / 256.0;
        const double rounds = floor(a_unit / 2.0), rest = a_unit - 2.0 * rounds;
        double computing = step * steps * (a_unit > 8.0 ? 0.78 * a_unit : 1.5 * rounds + (rest > 0.9 ? 1.5 : rest > 0.0 ? 1.0 : 0.0));
        const bool waits = a_unit > 2.0 || reading > computing;
        if (a_unit > 2.0) computing *= 1.0 - 0.15 * several;
        double us = cbrt(computing * computing * computing + reading * reading * reading) + (waits ? 0.35 * several * steps : 0.0) + 6.0 + (n > 1 ? 4.0 + call.merge_us * (double)n : 0.0);
        // (more than the places hold, where fewer would fill them: 4 contexts of up to 9000 keys 28.4, in a third of the pieces 24.2; of 30000 41.9, 36.7)
        if (a_unit > 2.0 && wgs < 256) us *= 1.0 + 0.05 * several;
        if (us < best.us) best = {(int32_t)n, us};
        return true;
    };
    for (int64_t p = 1; p <= kMaxPieces && consider(p); p += (p + 3) / 4) {}
    for (int64_t fill = 256; fill <= 512; fill += 256)                    // one workgroup a compute unit, two
        if (fill / wgs > 1) consider(fill / wgs);
    return best;
}

// Which kernel a call goes to: the one that is expected to be faster.
struct Choice { bool large; Plan plan; PagedLargePlan many; };
Choice choose(const kvs_shape *shape, const Paged &pg, float scale, size_t workspace_bytes)
{
    const PagedCall call = describe(shape, pg);
    Choice c;
    c.plan = plan_pieces(shape, pg, call, workspace_bytes);
    c.large = attention_paged_takes_large(shape, pg, call, scale, workspace_bytes, &c.many) && (c.many.us < c.plan.us || paged_forced_pieces);
    return c;
}

template <int DTYPE, int D, int PARTS>
kvs_status launch(const kvs_shape *shape, const kvs_paged_cache *c, const Paged &pg, int64_t units, const Plan &plan, const void *q, float scale,
                  void *out, float *lse_out, void *workspace, hipStream_t hs)
{
    static DeviceOnce once;
    constexpr int es = DTYPE == KVS_F32 ? 4 : 2;
    constexpr int lds = kWaves * 2 * kKeys * D * es;
    kvs_status st = once_per_device(once, [&]() -> kvs_status {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attention_paged_kernel<DTYPE, D, PARTS, false>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        return e == hipSuccess ? KVS_OK : fail(KVS_EHIP, "kvs_attention_paged: %s", hipGetErrorString(e));
    });
    if (st != KVS_OK) return st;
    const int64_t items = (int64_t)pg.n_new * shape->n_q_heads;
    const PagedParts parts = paged_parts(workspace, plan.pieces > 1 ? items * plan.pieces : 0);
    hipLaunchKernelGGL((attention_paged_kernel<DTYPE, D, PARTS, false>), dim3((unsigned)(units * plan.pieces * shape->n_kv_heads)), dim3(kThreads), lds, hs, pg, shape->n_q_heads,
                       shape->n_kv_heads, (int)units, plan.pieces, kLeastTiles, (const int32_t *)nullptr, (const char *)c->k, (const char *)c->v, q, scale * 1.4426950408889634f, out, lse_out, parts.o, parts.ml);
    if ((st = check_launch("kvs_attention_paged")) != KVS_OK || plan.pieces <= 1) return st;
    return launch_merge_paged(shape, pg, plan.pieces, parts, out, lse_out, hs);
}

} // namespace

kvs_status launch_merge_paged(const kvs_shape *shape, const Paged &pg, int pieces, const PagedParts &parts, void *out, float *lse_out, hipStream_t hs)
{
    const int64_t items = (int64_t)pg.n_new * shape->n_q_heads;
#define KVS_MERGE_ROWS(DT, DD, M)                                                                                                                              \
    hipLaunchKernelGGL((merge_paged_rows_kernel<DT, DD, M>), dim3((unsigned)((items + 4 * kThreads / DD - 1) / (4 * kThreads / DD))), dim3(kThreads), 0, hs, pg, items, \
                       shape->n_q_heads, pieces, parts.o, parts.ml, out, lse_out)
#define KVS_MERGE(DT, DD)                                                                                                                                      \
    do {                                                                                                                                                       \
        if (pieces <= 4) KVS_MERGE_ROWS(DT, DD, 4);                                                                                                            \
        else if (pieces <= 16 || items >= 1024) KVS_MERGE_ROWS(DT, DD, 16);                                                                                     \
        else hipLaunchKernelGGL((merge_paged_kernel<DT, DD>), dim3((unsigned)items, DD / 32), dim3(kThreads), 0, hs, pg, shape->n_q_heads, pieces, parts.o,    \
                                parts.ml, out, lse_out);                                                                                                       \
    } while (0)
    const bool wide = shape->head_dim == 128;
    if (shape->dtype == KVS_F32) { if (wide) KVS_MERGE(KVS_F32, 128); else KVS_MERGE(KVS_F32, 64); }
    else { if (wide) KVS_MERGE(KVS_BF16, 128); else KVS_MERGE(KVS_BF16, 64); }
#undef KVS_MERGE
#undef KVS_MERGE_ROWS
    return check_launch("kvs_attention_paged(merge)");
}

kvs_status launch_again_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const Paged &pg, const PagedLargePlan &plan, const int32_t *odd, const void *q, float scale,
                              void *out, float *lse_out, hipStream_t hs)
{
    static DeviceOnce once;
    constexpr int D = 128, lds = kWaves * 2 * kKeys * D * 2;
    const kvs_status st = once_per_device(once, [&]() -> kvs_status {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attention_paged_kernel<KVS_BF16, D, 1, true>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        return e == hipSuccess ? KVS_OK : fail(KVS_EHIP, "kvs_attention_paged: %s", hipGetErrorString(e));
    });
    if (st != KVS_OK) return st;
    hipLaunchKernelGGL((attention_paged_kernel<KVS_BF16, D, 1, true>), dim3((unsigned)(plan.units * shape->n_kv_heads)), dim3(kThreads), lds, hs, pg,
                       shape->n_q_heads, shape->n_kv_heads, (int)plan.units, plan.pieces, kLeastTiles, odd, (const char *)cache->k, (const char *)cache->v, q, scale * 1.4426950408889634f, out,
                       lse_out, (float *)nullptr, (float4 *)nullptr);
    return check_launch("kvs_attention_paged(again)");
}

size_t attention_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx, int64_t n_new)
{
    if (check_shape(shape) != KVS_OK || n_new <= 0 || max_ctx <= 0) return 256;
    const int64_t items = n_new * shape->n_q_heads;
    int64_t pieces = max_ctx / (kWaves * kKeys) + 2;
    if (pieces > kMaxPieces) pieces = kMaxPieces;
    const int64_t most = kMostCutWgs * kRows;                // rows of a cut launch's workgroups
    const int64_t slots = items < most && items * pieces < most ? items * pieces : most;
    size_t bytes = (size_t)slots * paged_slot_bytes(shape->head_dim);
    const size_t large = attention_paged_large_workspace_bytes(shape, batch, n_new);
    if (large > bytes) bytes = large;
    return (bytes + 255) / 256 * 256 + 256;
}

kvs_status check_paged(const char *me, const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages, Paged *out)
{
    kvs_status st = check_shape(shape);
    if (st != KVS_OK) return st;
    if (!cache || !pages) return fail(KVS_EINVAL, "%s: the cache or the page table is NULL", me);
    if (shape->n_kv_heads > 64) return fail(KVS_EUNSUPPORTED, "%s: more than 64 kv heads", me);
    if (shape->n_q_heads > 4096) return fail(KVS_EUNSUPPORTED, "%s: more than 4096 query heads", me);
    if (cache->page != 16 && cache->page != 32 && cache->page != 64 && cache->page != 128 && cache->page != 256)
        return fail(KVS_EINVAL, "%s: pages of %d rows (16, 32, 64, 128 and 256 are built)", me, cache->page);
    if (cache->n_pages < 0 || cache->n_pages > (int64_t)0x7fffffff / (cache->page / kGranule))
        return fail(KVS_EINVAL, "%s: %lld pages", me, (long long)cache->n_pages);
    if (pages->batch < 0 || pages->width < 0 || pages->max_ctx < 0) return fail(KVS_EINVAL, "%s: negative size of the page table", me);
    if (pages->max_ctx > 0x7fffff00LL) return fail(KVS_EINVAL, "%s: contexts of %lld rows", me, (long long)pages->max_ctx);
    if (pages->batch > 0 && (!pages->ctx_len || (pages->width > 0 && !pages->table))) return fail(KVS_EINVAL, "%s: the page table or the lengths are NULL", me);
    if (cache->n_pages > 0 && (!cache->k || !cache->v)) return fail(KVS_EINVAL, "%s: the cache's K or V is NULL", me);
    if (!aligned16(cache->k) || !aligned16(cache->v)) return fail(KVS_EINVAL, "%s: the cache's K and V must be 16-byte aligned", me);
    Paged pg = {};
    pg.table = pages->table;
    pg.ctx_len = pages->ctx_len;
    pg.batch = pages->batch;
    pg.width = pages->width;
    const int64_t rows = (int64_t)pages->width * cache->page;
    pg.max_ctx = (int32_t)(rows < pages->max_ctx ? rows : pages->max_ctx);
    if (cache->n_pages == 0) pg.max_ctx = 0;
    pg.n_pages = (int32_t)cache->n_pages;
    pg.page_log2 = __builtin_ctz((unsigned)cache->page);
    *out = pg;
    return KVS_OK;
}

kvs_status check_new_tokens(const char *me, const kvs_shape *shape, const kvs_page_table *pages, const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new,
                            int32_t window, int32_t n_first, Paged *out)
{
    if (n_new < 0) return fail(KVS_EINVAL, "%s: n_new < 0", me);
    if (window < 0 || n_first < 0) return fail(KVS_EINVAL, "%s: a negative window or number of first tokens", me);
    if (!cu_new && n_new != pages->batch) return fail(KVS_EINVAL, "%s: %lld tokens of %d requests without cu_new", me, (long long)n_new, pages->batch);
    if (n_new > 0x3fffff00LL / shape->n_q_heads) return fail(KVS_EINVAL, "%s: %lld tokens in one call", me, (long long)n_new);
    out->cu_new = cu_new;
    out->sel_pos = sel_pos;
    out->n_new = (int32_t)n_new;
    out->window = window;
    out->n_first = n_first;
    return KVS_OK;
}

} // namespace kvs

extern "C" kvs_status kvs_attention_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                          const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new, const void *q_new, float scale,
                                          int32_t window, int32_t n_first, void *out, float *lse_out,
                                          void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace kvs;
    const char *me = "kvs_attention_paged";
    Paged pg;
    kvs_status st = check_paged(me, shape, cache, pages, &pg);
    if (st != KVS_OK || (st = check_new_tokens(me, shape, pages, cu_new, sel_pos, n_new, window, n_first, &pg)) != KVS_OK) return st;
    if (!isfinite(scale * 1.4426950408889634f)) return fail(KVS_EINVAL, "%s: a scale of %g", me, (double)scale);
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(KVS_EINVAL, "%s: workspace must be 256-byte aligned", me);
    if (!workspace) workspace_bytes = 0;
    if (n_new == 0 || pages->batch == 0) return KVS_OK;
    if (!q_new || !out) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    if (!aligned16(q_new) || !aligned16(out)) return fail(KVS_EINVAL, "%s: Q/out pointers must be 16-byte aligned", me);
    const size_t heads = (size_t)n_new * shape->n_q_heads, bytes = heads * shape->head_dim * elem_bytes(shape->dtype);
    if (overlap(q_new, bytes, out, bytes)) return fail(KVS_EINVAL, "%s: out overlaps q_new", me);
    if (lse_out && (overlap(lse_out, heads * sizeof(float), q_new, bytes) || overlap(lse_out, heads * sizeof(float), out, bytes)))
        return fail(KVS_EINVAL, "%s: lse_out overlaps q_new or out", me);
    const size_t pool = pool_bytes(shape, cache), batch = (size_t)pages->batch;
    st = check_apart(me, {{out, bytes, "out"}, {lse_out, heads * sizeof(float), "lse_out"}},
                     {{cache->k, pool, "the cache's K"}, {cache->v, pool, "the cache's V"}, {pages->table, batch * pages->width * 4, "the page table"}, {pages->ctx_len, batch * 4, "ctx_len"},
                      {cu_new, (batch + 1) * 4, "cu_new"}, {sel_pos, (size_t)n_new * 4, "sel_pos"}});
    if (st != KVS_OK) return st;
    hipStream_t hs = (hipStream_t)stream;
    const int grp = shape->n_q_heads / shape->n_kv_heads;
    const Choice choice = choose(shape, pg, scale, workspace_bytes);
    if (choice.large) return launch_attention_paged_large(shape, cache, pg, choice.many, q_new, scale, out, lse_out, workspace, hs);
    const Plan &plan = choice.plan;
    const int64_t units = most_blocks(pg, grp, kRows);
    if (units * plan.pieces * shape->n_kv_heads > kMostWgs || (int64_t)pg.n_new * shape->n_q_heads * (plan.pieces > 1 ? 4 : 0) > kMostWgs)
        return fail(KVS_EINVAL, "%s: too many rows in one call", me);
    const bool wide = shape->head_dim == 128, few = (int64_t)pg.n_new * grp <= (int64_t)kRows * pg.batch;
#define KVS_AP(DT, DD, PP) launch<DT, DD, PP>(shape, cache, pg, units, plan, q_new, scale, out, lse_out, workspace, hs)
    if (shape->dtype == KVS_F32) {
        if (few) return wide ? KVS_AP(KVS_F32, 128, 2) : KVS_AP(KVS_F32, 64, 2);
        return wide ? KVS_AP(KVS_F32, 128, 1) : KVS_AP(KVS_F32, 64, 1);
    }
    if (few) return wide ? KVS_AP(KVS_BF16, 128, 2) : KVS_AP(KVS_BF16, 64, 2);
    return wide ? KVS_AP(KVS_BF16, 128, 1) : KVS_AP(KVS_BF16, 64, 1);
#undef KVS_AP
}

#ifdef KVS_PAGED_TEST
namespace kvs { int32_t paged_forced_pieces = 0; }

extern "C" KVS_API void kvs_test_force_pieces(int32_t pieces) { kvs::paged_forced_pieces = pieces; }

// What a call would do, without one (no tensor is read): whether it goes to the kernel of many rows, into how many pieces its keys are cut, whether
// row tiles are dealt there.
extern "C" KVS_API kvs_status kvs_test_choice(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages, const int32_t *cu_new, const int32_t *sel_pos,
                                              int64_t n_new, float scale, int32_t window, int32_t n_first, size_t workspace_bytes, int32_t *taken)
{
    using namespace kvs;
    Paged pg;
    kvs_status st = check_paged("kvs_test_choice", shape, cache, pages, &pg);
    if (st != KVS_OK || (st = check_new_tokens("kvs_test_choice", shape, pages, cu_new, sel_pos, n_new, window, n_first, &pg)) != KVS_OK) return st;
    const Choice c = choose(shape, pg, scale, workspace_bytes);
    taken[0] = c.large;
    taken[1] = c.large ? c.many.pieces : c.plan.pieces;
    taken[2] = c.large && c.many.dealt;
    return KVS_OK;
}
#endif
