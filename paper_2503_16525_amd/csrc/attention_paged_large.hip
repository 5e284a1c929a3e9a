// kvs_attention_paged with many rows a key: bf16, head_dim 128, 256 rows (tokens times query heads of a KV head) a workgroup.
//
// The same products as in attention_paged.hip, S^T = K Q^T and O^T += V^T P^T, but 64 rows a wave: every 16 bytes of K or V that a
// lane reads from LDS feed two matrix instructions, and a tile that is loaded once serves 256 rows.  The accumulators, Q and
// two score tiles take the whole register file, so one wave a SIMD is resident and works on three tiles at once: in step j, the
// scores of tile j + 1, the weights of tile j and the product of tile j - 1 with V, eight slices of four matrix instructions with
// vector work beside each.
//
// Tiles.  A workgroup's tiles are numbered along what its rows see: `head` tiles of first tokens, then those from `low` on.  Where
// their rows are is looked up once, into LDS (two runs of 16 rows a tile), so that a step reads two numbers and has two addresses.
// K and V go straight into LDS, rings of four and eight tiles; a tile is asked for four steps ahead, and the one barrier of a
// step is where each wave waits for its own loads of the tile after next.
//
// The softmax's reference is the largest score of a row's first tile, and moves only where a sum passes 2^64, to 3 above the tile's largest score or by 66 if
// that is more: then the tile's weights, which have not met V yet, are made again, and sums and accumulators come down with it.  So a row's largest
// weight is never far below 1: products with a V down to 2^-100 keep their bits, and of two pieces whose references are so far apart that the merge gives one of them
// nothing, that one had nothing to give (at 2^-58 of the other's weight).  Raised above the first scores by 60, as weights would allow, neither held: V
// of 2^-70 lost bits, V of 2^-90 was 0, and pieces with a quarter of another's weight were lost.  A row that has seen nothing yet has the lowest reference and a sum
// of 0, so that its first score moves it.
//
// A weight of 0 does not hide a V that is infinite or NaN.  A workgroup whose sums are no numbers, or that met an entry of the table
// that names no page, says so, and a last launch does its rows once more with the kernel of attention_paged.hip, which
// multiplies such keys with the weights of the rows that see them.  (Almost always nothing is to do: 4 us.)
//
// What bounds it: vector instructions and matrix instructions, of which a step has 32 and about 200 others, that hide each other by half, at a clock that comes
// down as they do (2.08 GHz at 41 % of the matrix pipes' cycles, 1.9 to 1.98 at 47 %).  2048 tokens of 32 heads over 32768 keys 978 to 985 us by box, 1.08 to
// 1.09 PFLOP/s; 8192 under a window of 4096 427 to 433, 0.95 to 0.97.  Weights meet V as one bf16 number: of the output's norm 0.0023 and 0.0020 are errors
// there, 0.0017 and 0.0015 from rounding the output alone; a second number would be 48 matrix instructions a step for 32.  On the first: all but the scores' products left out 897, no exponentials 857, nothing read or
// loaded 841.  v_dot2 shares the matrix pipes: shifts and additions in its place 997, no sum of the rounded weights at all 937, which would cost a row that
// one key dominates its exactness.  Operands asked for two slices ahead, weights in seven slices of eight, and a check every other step gained nothing.
#include "attention_paged.h"

#include <type_traits>

namespace kvs {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

constexpr int D = 128;
constexpr int BN = 32;                 // keys of a tile
constexpr int NWAVES = 4, NT = NWAVES * kWave;
constexpr int NB = 2;                  // blocks of 32 rows a wave
constexpr int ROWS = NWAVES * 32 * NB;
static_assert(ROWS == kPagedLargeRows, "");
constexpr int ROW_B = D * 2, TILE_B = BN * ROW_B;
constexpr int AHEAD = 4;               // steps between a tile's request and its weights
constexpr int K_RING = 4, V_RING = 8;
constexpr int RING_B = (K_RING + V_RING) * TILE_B;
constexpr int PLACES_AT = RING_B + 48;
constexpr int kMostTiles = 6144;       // of a piece: 48 KB of places
constexpr int kLeastTiles = 8;         // of a piece
constexpr int kMostPieces = 32, kMostCutWgs = 512;
constexpr float kSumLimit = 1.8446744e19f;   // 2^64

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// acc + lo(w) + hi(w): the normaliser is made of the rounded weights, so that numerator and denominator carry the same rounding
__device__ __forceinline__ float add_rounded_pair(uint32_t w, float acc)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), acc, false);
}

template <bool DEALT>
__global__ __launch_bounds__(NT, 1) void attention_paged_large_kernel(
    const Paged pg, int n_q_heads, int n_kv_heads, int units, int pieces, int least_tiles, const char *__restrict__ k_pool, const char *__restrict__ v_pool,
    const uint16_t *__restrict__ q_new, float scale_log2, uint16_t *__restrict__ out, float *__restrict__ lse_out, float *__restrict__ part_o, float4 *__restrict__ part_ml, int32_t *__restrict__ odd_out)
{
    extern __shared__ __attribute__((aligned(16))) char lds_b[];         // rings of K and V; meet_s, odd_s; places
    int (*const meet_s)[2] = reinterpret_cast<int (*)[2]>(lds_b + RING_B);
    int &odd_s = *reinterpret_cast<int *>(lds_b + RING_B + sizeof(int[NWAVES][2]));

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hf = lane >> 5, ln = lane & 31;
    // Workgroup = (piece, row tile, KV head); the last row tiles, which see most, begin.
    const int grp = n_q_heads / n_kv_heads;
    // DEALT: a workgroup for every compute unit, which takes the row tiles of one KV head in turn, there and back, the longest first.
    const PagedPlace at = DEALT ? PagedPlace{0, (int)(blockIdx.x % (uint32_t)n_kv_heads), (int)(blockIdx.x / (uint32_t)n_kv_heads)} : place_of(blockIdx.x, units, pieces, n_kv_heads);
    const int g = __builtin_amdgcn_readfirstlane(at.g), piece = __builtin_amdgcn_readfirstlane(at.piece), at_unit = __builtin_amdgcn_readfirstlane(at.unit);
    const int lanes = DEALT ? (int)(gridDim.x / (uint32_t)n_kv_heads) : 0;
    for (int round = 0; round == 0 || DEALT; ++round) {
    const int unit = !DEALT ? at_unit : round * lanes + (round & 1 ? lanes - 1 - at_unit : at_unit);
    if (DEALT && unit >= units) return;
    if (DEALT && round) __syncthreads();
    int32_t *const odd_at = odd_out + ((int64_t)piece * units + unit) * n_kv_heads + g;
    Block mine;
    if (!find_block<ROWS>(pg, grp, units - 1 - unit, mine)) {
        if (tid == 0) *odd_at = 0;
        if (DEALT) continue;
        return;
    }
    const int b = __builtin_amdgcn_readfirstlane(mine.b), blk = __builtin_amdgcn_readfirstlane(mine.blk), tok0 = __builtin_amdgcn_readfirstlane(mine.tok0);
    const int n_tok = __builtin_amdgcn_readfirstlane(mine.n_tok), len = __builtin_amdgcn_readfirstlane(mine.len), end = __builtin_amdgcn_readfirstlane(mine.end);
    const int rows = n_tok * grp;
    // Row tiles end with their request's rows: the one partly filled is the first, whose rows see least.
    const int row0 = blk * ROWS - ((rows + ROWS - 1) / ROWS * ROWS - rows);
    // A wave has one of the four lower blocks of 32 rows and its counterpart among the upper ones.
    auto block_row = [&](int nb) { return 32 * (nb == 0 ? wave : 2 * NWAVES - 1 - wave); };

    const int window = pg.window, n_first = window ? pg.n_first : 0;
    bool row_ok[NB];
    int pos[NB];
    int64_t row_idx[NB];
    int pmin = 0x7fffffff, pmax = -1, plow = 0x7fffffff;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int rq = row0 + block_row(nb) + ln;
        row_ok[nb] = rq >= 0;
        const int t = max(rq, 0) / grp;
        pos[nb] = position_of(pg, tok0, n_tok, t, len, end);
        row_idx[nb] = (int64_t)(tok0 + t) * n_q_heads + g * grp + (max(rq, 0) - t * grp);
        pmin = min(pmin, pos[nb]);
        pmax = max(pmax, pos[nb]);
        plow = min(plow, pos[nb] < 0 ? 0x7fffffff : pos[nb]);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        pmin = min(pmin, __shfl_xor(pmin, o));
        pmax = max(pmax, __shfl_xor(pmax, o));
        plow = min(plow, __shfl_xor(plow, o));
    }
    pmin = __builtin_amdgcn_readfirstlane(pmin);
    pmax = __builtin_amdgcn_readfirstlane(pmax);
    if (lane == 0) { meet_s[wave][0] = pmax; meet_s[wave][1] = plow; }
    if (tid == 0) odd_s = 0;

    u32x4_t qreg[NB][D / 16];          // Q as the B operand
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qreg[nb][ks] = *reinterpret_cast<const u32x4_t *>(q_new + row_idx[nb] * D + 16 * ks + 8 * hf);
    // only ever an operand of matrix instructions: kept in the accumulation half of the register file
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+a"(qreg[nb][ks]));

    __syncthreads();
    int wg_pmax = -1, wg_plow = 0x7fffffff;
#pragma unroll
    for (int w = 0; w < NWAVES; ++w) { wg_pmax = max(wg_pmax, meet_s[w][0]); wg_plow = min(wg_plow, meet_s[w][1]); }
    wg_pmax = __builtin_amdgcn_readfirstlane(wg_pmax);
    wg_plow = __builtin_amdgcn_readfirstlane(wg_plow);
    const int low = window && wg_pmax >= 0 ? max(wg_plow - window + 1, 0) / BN : 0;
    const int head = min(low, (int)(((int64_t)n_first + BN - 1) / BN));
    const int total = wg_pmax < 0 ? 0 : head + wg_pmax / BN + 1 - low;
    const int piece_tiles = max((total + pieces - 1) / pieces, least_tiles);
    const int t_lo = (int)min((int64_t)piece * piece_tiles, (int64_t)total), t_hi = (int)min((int64_t)t_lo + piece_tiles, (int64_t)total);
    auto tile_of = [&](int t) { return t < head ? t : t - head + low; };
    if (t_lo >= t_hi) {                                      // nothing to see here
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if (!row_ok[nb]) continue;
            if (pieces > 1) {
                if (hf == 0) part_ml[row_idx[nb] * pieces + piece] = make_float4(kLowest, 0.f, 0.f, 0.f);
            } else {
#pragma unroll
                for (int c = 0; c < D / 16; ++c) *reinterpret_cast<uint4 *>(out + row_idx[nb] * D + 16 * c + 8 * hf) = make_uint4(0u, 0u, 0u, 0u);
                if (lse_out && hf == 0) lse_out[row_idx[nb]] = -INFINITY;
            }
        }
        if (tid == 0) *odd_at = 0;
        if (DEALT) continue;
        return;
    }

    // ---- places of the piece's tiles, two runs of 16 rows each; behind the context its last run --------------------------
    int *const place_s = reinterpret_cast<int *>(lds_b + PLACES_AT);
    const int last_run = (len - 1) / kGranule;
    bool odd = false;                                        // a run of no page
    for (int e = tid; e < 2 * (t_hi - t_lo); e += NT) {
        const int run = granule_of(pg, b, min(2 * tile_of(t_lo + (e >> 1)) + (e & 1), last_run));
        odd = odd || run < 0;
        place_s[e] = max(run, 0);
    }
    if (odd) odd_s = 1;

    // ---- staging ------------------------------------------------------------------------------------------------------
    // One instruction moves 64 x 16 bytes, four rows, to 1 KiB of LDS.  Waves 0 and 1 stage the first and the second run of a tile's K, waves 2
    // and 3 those of V: a wave has one address a step.  Piece p of row r lies at p ^ f(r): f = r & 15 for K (8 lanes read one piece of 8 rows),
    // 2 (r & 7) for V (a transposing read covers 4 rows x 2 pieces).
    const uint32_t row_bytes = (uint32_t)n_kv_heads * ROW_B;
    const uint64_t run_bytes = (uint64_t)row_bytes * kGranule;
    const bool of_k = wave < 2;
    // (the select is one of scalars, which the compiler has to be told)
    const uint64_t st_pool = (uint64_t)(of_k ? k_pool : v_pool) + (uint32_t)g * ROW_B;
    const char *const st_head = (const char *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)st_pool) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(st_pool >> 32)) << 32);
    const int st_mask = of_k ? K_RING - 1 : V_RING - 1;
    const uint32_t st_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds_b) +
                             (uint32_t)((of_k ? 0 : K_RING) * TILE_B + (wave & 1) * kGranule * ROW_B);
    uint32_t st_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * i + (lane >> 4);
        st_off[i] = (uint32_t)r * row_bytes + (uint32_t)((lane & 15) ^ (of_k ? r : 2 * (r & 7))) * 16u;
    }
    auto load_1k = [&](uint32_t dst, uint32_t off, const char *base) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst), "v"(off), "s"(base) : "memory");
    };
    // Tile t goes to K slot t % K_RING and V slot t % V_RING, in the second half of step t - AHEAD, behind that step's barrier: the
    // slots' former tiles were last read a step before it at the latest.  Tiles behind the piece's last are loads of
    // that one, which nothing reads: the number of loads in flight is the same in every step.
    auto run_of = [&](int t) -> int { return __builtin_amdgcn_readfirstlane(place_s[2 * (min(max(t, t_lo), t_hi - 1) - t_lo) + (wave & 1)]); };
    auto stage_part = [&](int t, int part, int run) {
        load_1k(st_base + (uint32_t)((t & st_mask) * TILE_B + part * 4 * ROW_B), st_off[part], st_head + (uint64_t)(uint32_t)run * run_bytes);
    };
    auto stage_tile = [&](int t) {
        const int run = run_of(t);
#pragma unroll
        for (int part = 0; part < 4; ++part) stage_part(t, part, run);
    };
#define KVS_PAGED_BARRIER(in_flight) asm volatile("s_waitcnt vmcnt(" #in_flight ")\n\ts_barrier" ::: "memory")

    // ---- operands -----------------------------------------------------------------------------------------------------
    // K rows are fed with bits 2 and 3 swapped, so that entry r of a lane's scores is key 16 (r >> 3) + 8 hf + (r & 7).  V's operand, 8 keys
    // of a channel, comes out of two transposing reads (attention_paged.hip).
    const int krow = (ln & ~12) | ((ln & 4) << 1) | ((ln & 8) >> 1);
    const uint32_t k_read = (uint32_t)(krow * ROW_B + ((hf ^ (krow & 15)) * 16));
    const int tr_s = lane & 15, tr_g = lane >> 4;
    const int tr_key = 8 * (tr_g >> 1) + (tr_s >> 2), tr_c = 2 * (tr_g & 1) + ((tr_s & 3) >> 1);
    const uint32_t v_read_lo = (uint32_t)(tr_key * ROW_B + ((tr_c ^ (2 * (tr_key & 7))) * 16) + 8 * (tr_s & 1));
    const uint32_t v_read_hi = (uint32_t)((tr_key + 4) * ROW_B + ((tr_c ^ (2 * ((tr_key + 4) & 7))) * 16) + 8 * (tr_s & 1));
    // (Addresses in LDS are numbers: the rings begin at 0, the kernel has no other LDS, and every offset that is not the lane's is in bits that the
    // lane's part leaves 0, so that one instruction makes an address of both.)
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
    auto read_k = [&](uint32_t slot, int ks) -> u32x4_t { return *(const lds_u32x4 *)(uintptr_t)(k_read ^ ((uint32_t)(32 * ks) | slot)); };
    auto read_vt = [&](uint32_t slot, int a, int db) -> u32x4_t {
        typedef short v4i16 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(uintptr_t)((v_read_lo ^ ((uint32_t)(64 * db) | slot)) + 16 * a * ROW_B)));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(uintptr_t)((v_read_hi ^ ((uint32_t)(64 * db) | slot)) + 16 * a * ROW_B)));
        return u32x4_t{lo.x, lo.y, hi.x, hi.y};
    };
    auto k_slot = [&](int t) -> uint32_t { return (uint32_t)((t & (K_RING - 1)) * TILE_B); };
    auto v_slot = [&](int t) -> uint32_t { return (uint32_t)((K_RING + (t & (V_RING - 1))) * TILE_B); };
    const floatx16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto qk = [&](int t, floatx16 (&s)[NB]) {
        const uint32_t slot = k_slot(t);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const u32x4_t a = read_k(slot, ks);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qreg[nb][ks]), ks == 0 ? zero : s[nb], 0, 0, 0);
        }
    };

    // ---- masks: a bit for each key of a tile, from the lane's first (8 hf) on; entry r is bit 16 (r >> 3) + (r & 7) ---------------
    // (A bit spread over a word and a bitwise choice: no comparison results to be kept in scalar registers.)
    int upto[NB], below[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        upto[nb] = pos[nb] - 8 * hf;
        below[nb] = (window ? max(pos[nb] - window, -1) : -1) - 8 * hf;
    }
    const int first_end = n_first - 8 * hf;
    auto bits_below = [](int n) -> uint32_t { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };
    auto seen_bits = [&](int nb, int x0) -> uint32_t {
        const uint32_t first = first_end <= x0 ? 0u : bits_below(first_end - x0);
        return bits_below(upto[nb] - x0 + 1) & (~bits_below(below[nb] - x0 + 1) | first);
    };
    auto masked_score = [](float x, uint32_t bits, int r) -> float {
        const uint32_t seen = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 16 * (r >> 3) + (r & 7), 1);
        return __uint_as_float((__float_as_uint(x) & seen) | (0xff800000u & ~seen));
    };
    // tiles clear_lo .. clear_hi - 1 are seen whole by all rows of the wave
    const int clear_lo = window ? head + max(pmax - window < 0 ? 0 : (pmax - window) / BN + 1 - low, 0) : 0, clear_hi = pmin < 0 ? 0 : head + (pmin + 1) / BN - low;
    auto mask_tile = [&](int t, floatx16 (&s)[NB]) {
        const int x0 = tile_of(t) * BN;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const uint32_t bits = seen_bits(nb, x0);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[nb][r] = masked_score(s[nb][r], bits, r);
        }
    };
    auto row_max = [&](const floatx16 &s) -> float {         // of a row's scores, in powers of two
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        return fmaxf(mx, __shfl_xor(mx, 32)) * scale_log2;
    };

    floatx16 o_acc[D / 32][NB];
    float m_ref[NB], l_run[NB];                              // reference; this half-wave's share of the sum of rounded weights
    // and of the unrounded ones: l_exact is one tile's, added with the rounding error carried along
    float l_exact[NB], l_before[NB], le_before[NB], le_carry[NB];
    auto softmax4 = [&](const floatx16 &s, int nb, int r0, u32x4_t (&pop)[2]) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[r0 + 0], scale_log2, -m_ref[nb]));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[r0 + 1], scale_log2, -m_ref[nb]));
        const float e2 = __builtin_amdgcn_exp2f(fmaf(s[r0 + 2], scale_log2, -m_ref[nb]));
        const float e3 = __builtin_amdgcn_exp2f(fmaf(s[r0 + 3], scale_log2, -m_ref[nb]));
        const uint32_t w0 = pack2(e0, e1), w1 = pack2(e2, e3);
        pop[r0 >> 3][(r0 & 7) >> 1] = w0;
        pop[r0 >> 3][((r0 & 7) >> 1) + 1] = w1;
        l_run[nb] = add_rounded_pair(w1, add_rounded_pair(w0, l_run[nb]));
        l_exact[nb] += (e0 + e1) + (e2 + e3);
    };
    auto keep_sums = [&]() {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            l_before[nb] = l_run[nb];
            const float y = l_exact[nb] - le_carry[nb], sum = le_before[nb] + y;
            le_carry[nb] = (sum - le_before[nb]) - y;
            le_before[nb] = sum;
            l_exact[nb] = 0.f;
        }
    };
    auto outgrown = [&]() __attribute__((always_inline)) -> bool { return __builtin_amdgcn_ballot_w64(fmaxf(l_run[0], l_run[1]) >= kSumLimit) != 0; };
    auto recentre = [&](int t, floatx16 (&s)[NB], u32x4_t (&pop)[NB][2]) __attribute__((always_inline)) {
        mask_tile(t, s);                  // (the scores are not read again)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            floatx16 &m = s[nb];
            const float other = __shfl_xor(l_run[nb], 32);
            const bool move = l_run[nb] >= kSumLimit || other >= kSumLimit;
            // (A sum of up to 2^64 that comes down by more than 2^126, where the exponential makes it 0, is below 2^-59 of the tile's largest
            // weight.  A sum can also pass 2^64 by a weight of little more than nothing.  0 and 64 would do as well: 2048 tokens over 32768 keys 1016 us
            // for 985, by how the compiler orders the whole kernel.)
            const float to = move ? fmaxf(row_max(m) + 3.f, m_ref[nb] + 66.f) : m_ref[nb];
            const float down = move ? __builtin_amdgcn_exp2f(m_ref[nb] - to) : 1.f;
            m_ref[nb] = to;
            l_run[nb] = l_before[nb] * down;
            le_before[nb] *= down;
            le_carry[nb] *= down;
            l_exact[nb] = 0.f;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o_acc[db][nb][r] *= down;
#pragma unroll
            for (int r0 = 0; r0 < 16; r0 += 4) softmax4(m, nb, r0, pop[nb]);
        }
    };

    // One step: scores of tile jt + 1, weights of tile jt, product of tile jt - 1.  On entry the tiles jt - 1 .. jt + 1 are in the rings
    // and jt + 2, jt + 3 on their way; s_in holds tile jt's scores, p_in tile jt - 1's weights, ka and va slice 0's operands.
    auto step = [&](auto masked, int jt, floatx16 (&s_in)[NB], floatx16 (&s_out)[NB], const u32x4_t (&p_in)[NB][2], u32x4_t (&p_out)[NB][2], u32x4_t &ka, u32x4_t &va,
                    int &run) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked)::value;
        keep_sums();
        const uint32_t ks = k_slot(jt + 1), vs = v_slot(jt - 1), ks_next = k_slot(jt + 2), vs_next = v_slot(jt);
        uint32_t bits[NB] = {};
        if (MASKED) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) bits[nb] = seen_bits(nb, tile_of(jt) * BN);
        }
        const int now = run;
        run = run_of(jt + AHEAD + 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u32x4_t ka_n, va_n;
            if (i < 7) {
                ka_n = read_k(ks, i + 1);
                va_n = read_vt(vs, (i + 1) >> 2, (i + 1) & 3);
            } else {
                ka_n = read_k(ks_next, 0);
                va_n = read_vt(vs_next, 0, 0);
            }
            const int nbs = i >> 2, r0 = 4 * (i & 3), a = i >> 2, db = i & 3;
            s_out[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(ka), as_bf16x8(qreg[0][i]), i == 0 ? zero : s_out[0], 0, 0, 0);
            float x[4], e[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = fmaf(s_in[nbs][r0 + u], scale_log2, -m_ref[nbs]);
            if (MASKED) {
#pragma unroll
                for (int u = 0; u < 4; ++u) x[u] = masked_score(x[u], bits[nbs], r0 + u);
            }
            s_out[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(ka), as_bf16x8(qreg[1][i]), i == 0 ? zero : s_out[1], 0, 0, 0);
#pragma unroll
            for (int u = 0; u < 4; ++u) e[u] = __builtin_amdgcn_exp2f(x[u]);
            o_acc[db][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(va), as_bf16x8(p_in[0][a]), o_acc[db][0], 0, 0, 0);
#pragma unroll
            for (int u = 0; u < 4; u += 2) p_out[nbs][r0 >> 3][((r0 & 7) + u) >> 1] = pack2(e[u], e[u + 1]);
#pragma unroll
            for (int u = 0; u < 4; u += 2) l_run[nbs] = add_rounded_pair(p_out[nbs][r0 >> 3][((r0 & 7) + u) >> 1], l_run[nbs]);
            l_exact[nbs] += (e[0] + e[1]) + (e[2] + e[3]);
            o_acc[db][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(va), as_bf16x8(p_in[1][a]), o_acc[db][1], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);               // a slice's vector work stays beside its products (without: all products first, 1073 -> 991 us)
            ka = ka_n;
            va = va_n;
            if (i == 3) KVS_PAGED_BARRIER(4);                // tile jt + 2 has landed; jt + 3 may be in flight
            if (i >= 4) stage_part(jt + AHEAD, i - 4, now);
        }
        asm volatile("" : "+v"(l_exact[0]), "+v"(l_exact[1]));       // (not put off to the branch below)
        if (outgrown()) recentre(jt, s_in, p_out);
    };
    auto product = [&](int t, const u32x4_t (&pop)[NB][2]) {
        const uint32_t slot = v_slot(t);
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                const u32x4_t va = read_vt(slot, a, db);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) o_acc[db][nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(va), as_bf16x8(pop[nb][a]), o_acc[db][nb], 0, 0, 0);
            }
    };

    // ---- the sweep ----------------------------------------------------------------------------------------------------
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) l_run[nb] = l_exact[nb] = l_before[nb] = le_before[nb] = le_carry[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) o_acc[db][nb] = zero;
    __syncthreads();                                         // the places are there
    // Steps come in pairs.  The first tile takes none; of an even number of tiles a copy of the first comes before it, whose weights are 0.
    const int begin = t_lo - (1 - ((t_hi - t_lo) & 1));
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) stage_tile(begin + k);
    KVS_PAGED_BARRIER(0);
    {
        floatx16 s_cur[NB], s_nxt[NB];
        u32x4_t p_a[NB][2], p_b[NB][2];
        qk(begin, s_cur);
        mask_tile(t_lo, s_cur);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float top = row_max(s_cur[nb]);
            m_ref[nb] = top > kLowest ? top : kLowest;       // (NaN: the lowest, and the weights say so)
#pragma unroll
            for (int r = 0; r < 16; ++r) s_cur[nb][r] = begin < t_lo ? -INFINITY : s_cur[nb][r];
        }
        qk(begin + 1, s_nxt);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int r0 = 0; r0 < 16; r0 += 4) softmax4(s_cur[nb], nb, r0, p_a[nb]);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");          // (K of the first tile has been read)
        stage_tile(begin + AHEAD);
        u32x4_t ka = read_k(k_slot(begin + 2), 0), va = read_vt(v_slot(begin), 0, 0);
        int run = run_of(begin + 1 + AHEAD);
        int jt = begin + 1;
        // two steps a trip, so that scores and weights swap roles without copies
        auto sweep = [&](auto masked, int stop) __attribute__((always_inline)) {
            for (; jt < stop && jt + 1 < t_hi; jt += 2) {
                step(masked, jt, s_nxt, s_cur, p_a, p_b, ka, va, run);
                step(masked, jt + 1, s_cur, s_nxt, p_b, p_a, ka, va, run);
            }
        };
        sweep(std::true_type{}, clear_lo);
        sweep(std::false_type{}, clear_hi - 1);
        sweep(std::true_type{}, t_hi);
        // The last tile's V meets its weights here: rows behind the context, which may hold anything, become 0 before it does.
        const int x0 = tile_of(t_hi - 1) * BN;
        if (x0 + BN > len) {
            __syncthreads();
            for (int key = wave; key < BN; key += NWAVES)
                if (x0 + key >= len) *reinterpret_cast<uint32_t *>(lds_b + v_slot(t_hi - 1) + key * ROW_B + 4 * lane) = 0u;
            __syncthreads();
        }
        product(t_hi - 1, p_a);
        keep_sums();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // nothing may be on its way into LDS when the workgroup ends

    float l_tot[NB], le_tot[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l_tot[nb] = l_run[nb] + __shfl_xor(l_run[nb], 32);
        const float e = le_before[nb] - le_carry[nb];
        le_tot[nb] = e + __shfl_xor(e, 32);
    }
    {
        float sum = 0.f;                                     // 0, or NaN
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum = fmaf(o_acc[db][nb][r], 0.f, sum);
        if (!(sum == 0.f)) odd_s = 1;
    }
    __syncthreads();
    if (tid == 0) *odd_at = odd_s;

    // ---- what comes out -----------------------------------------------------------------------------------------------
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        if (!row_ok[nb]) continue;
        if (pieces > 1) {
            const int64_t slot = row_idx[nb] * pieces + piece;
            if (hf == 0) part_ml[slot] = make_float4(m_ref[nb], le_tot[nb], l_tot[nb], 0.f);
            if (le_tot[nb] == 0.f) continue;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4)
                    *reinterpret_cast<float4 *>(part_o + slot * D + 32 * db + 8 * r4 + 4 * hf) =
                        make_float4(o_acc[db][nb][4 * r4], o_acc[db][nb][4 * r4 + 1], o_acc[db][nb][4 * r4 + 2], o_acc[db][nb][4 * r4 + 3]);
            continue;
        }
        const float inv = le_tot[nb] != 0.f ? 1.f / l_tot[nb] : 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<uint2 *>(out + row_idx[nb] * D + 32 * db + 8 * r4 + 4 * hf) =
                    make_uint2(pack2(o_acc[db][nb][4 * r4] * inv, o_acc[db][nb][4 * r4 + 1] * inv), pack2(o_acc[db][nb][4 * r4 + 2] * inv, o_acc[db][nb][4 * r4 + 3] * inv));
        if (lse_out && hf == 0) lse_out[row_idx[nb]] = le_tot[nb] != 0.f ? (m_ref[nb] + log2f(le_tot[nb])) * 0.69314718055994531f : -INFINITY;
    }
    }   // row tiles
}

inline size_t odd_bytes(int64_t wgs) { return ((size_t)wgs * 4 + 255) / 256 * 256; }

} // namespace

size_t attention_paged_large_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t n_new)
{
    if (shape->dtype != KVS_BF16 || shape->head_dim != D) return 0;
    const int64_t items = n_new * shape->n_q_heads, most = (int64_t)kMostCutWgs * ROWS;
    const int64_t most_units = n_new * (shape->n_q_heads / shape->n_kv_heads) / ROWS + (batch < n_new ? batch : n_new) * (1 + shape->n_q_heads / shape->n_kv_heads / ROWS);
    const int64_t slots = items < most && items * kMostPieces < most ? items * kMostPieces : most;
    return (size_t)slots * paged_slot_bytes(D) + odd_bytes(most_units * kMostPieces * shape->n_kv_heads);
}

bool attention_paged_takes_large(const kvs_shape *shape, const Paged &pg, const PagedCall &call, float scale, size_t workspace_bytes, PagedLargePlan *plan)
{
    if (shape->dtype != KVS_BF16 || shape->head_dim != D || !(scale > 0.f) || scale > 3.0e37f || pg.max_ctx == 0) return false;
    const int64_t units = most_blocks(pg, call.grp, ROWS);
    int64_t keys = pg.max_ctx;
    if (pg.window && !pg.sel_pos) {                          // consecutive tokens: the window, and what 256 rows lie apart
        const int64_t some = (int64_t)pg.window + ROWS / (call.grp < ROWS ? call.grp : ROWS) + 2 * BN + pg.n_first + BN;
        if (some < keys) keys = some;
    }
    const int64_t tiles = (keys + BN - 1) / BN + 1, wgs = (int64_t)call.row_tiles * pg.batch * shape->n_kv_heads;
    if (workspace_bytes < odd_bytes(units * shape->n_kv_heads)) return false;
    auto fits = [&](int64_t p) { return odd_bytes(units * p * shape->n_kv_heads) + (size_t)(call.items * p) * paged_slot_bytes(D) <= workspace_bytes; };
    plan->us = 1e30;
    for (int64_t p = 1; p <= kMostPieces && (p == 1 || (fits(p) && wgs * p <= kMostCutWgs)); ++p) {
        const int64_t each = (tiles + p - 1) / p;
        if (each > kMostTiles || (paged_forced_pieces && p != paged_forced_pieces)) continue;
        if (p > 1 && each < kLeastTiles) break;
        // Rounds of one workgroup a compute unit: 0.90 us a tile and 6 to begin and end; 3 for the last launch; a merge.  (us, estimate and
        // measured: 256 tokens of 32 heads over 16384 keys in one piece 471, 437; eight 91, 93; ten 139, 134; 500 of 28 heads over 12000 in four 115, 113.)
        const double us = (double)((wgs * p + 255) / 256) * (0.90 * (double)each + 6.0) + 3.0 + (p > 1 ? 4.0 + call.merge_us * (double)p : 0.0);
        if (us < plan->us) {
            plan->us = us;
            plan->pieces = (int32_t)p;
        }
    }
    if (plan->us == 1e30 || units * plan->pieces * shape->n_kv_heads > kMostWgs) return false;
    plan->tiles = (int32_t)((tiles + plan->pieces - 1) / plan->pieces);
    plan->units = units;
    // (The rows of one request: of several, whose contexts differ, every tile finds its place as one becomes free.)
    plan->dealt = plan->pieces == 1 && pg.batch == 1 && units * shape->n_kv_heads > 256 && 256 % shape->n_kv_heads == 0;
    return true;
}

kvs_status launch_attention_paged_large(const kvs_shape *shape, const kvs_paged_cache *cache, const Paged &pg, const PagedLargePlan &plan, const void *q, float scale,
                                        void *out, float *lse_out, void *workspace, hipStream_t hs)
{
    static DeviceOnce once;
    constexpr int most_lds = PLACES_AT + 8 * kMostTiles;
    kvs_status st = once_per_device(once, [&]() -> kvs_status {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attention_paged_large_kernel<false>), hipFuncAttributeMaxDynamicSharedMemorySize, most_lds);
        if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attention_paged_large_kernel<true>), hipFuncAttributeMaxDynamicSharedMemorySize, most_lds);
        hipFuncAttributes one = {}, other = {};
        if (e == hipSuccess) e = hipFuncGetAttributes(&one, reinterpret_cast<const void *>(&attention_paged_large_kernel<false>));
        if (e == hipSuccess) e = hipFuncGetAttributes(&other, reinterpret_cast<const void *>(&attention_paged_large_kernel<true>));
        if (e == hipSuccess && one.sharedSizeBytes + other.sharedSizeBytes != 0) return fail(KVS_EHIP, "kvs_attention_paged: its rings do not begin at address 0");
        return e == hipSuccess ? KVS_OK : fail(KVS_EHIP, "kvs_attention_paged: %s", hipGetErrorString(e));
    });
    if (st != KVS_OK) return st;
    const int64_t wgs = plan.units * plan.pieces * shape->n_kv_heads;
    int32_t *const odd = (int32_t *)workspace;
    const PagedParts parts = paged_parts((char *)workspace + odd_bytes(wgs), (int64_t)pg.n_new * shape->n_q_heads * plan.pieces);
    const int lds = PLACES_AT + (8 * plan.tiles + 15) / 16 * 16;
#define KVS_LARGE(DEAL, N)                                                                                                                                      \
    hipLaunchKernelGGL(attention_paged_large_kernel<DEAL>, dim3((unsigned)(N)), dim3(NT), lds, hs, pg, shape->n_q_heads, shape->n_kv_heads, (int)plan.units,    \
                       plan.pieces, plan.tiles < kLeastTiles ? plan.tiles : kLeastTiles, (const char *)cache->k, (const char *)cache->v, (const uint16_t *)q,   \
                       scale * 1.4426950408889634f, (uint16_t *)out, lse_out, parts.o, parts.ml, odd)
    if (plan.dealt) KVS_LARGE(true, 256);
    else KVS_LARGE(false, wgs);
#undef KVS_LARGE
    if ((st = check_launch("kvs_attention_paged")) != KVS_OK) return st;
    if (plan.pieces > 1 && (st = launch_merge_paged(shape, pg, plan.pieces, parts, out, lse_out, hs)) != KVS_OK) return st;
    return launch_again_paged(shape, cache, pg, plan, odd, q, scale, out, lse_out, hs);
}

} // namespace kvs
