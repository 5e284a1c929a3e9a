// kvs_mass_paged: the attention that every cached row receives from a call's tokens, added to what it received before.
//
// Mathematics.  mass[i] += sum over rows r (tokens times the query heads of the KV head) of exp(scale q_r . k_i - lse_r): the column sums
// of a softmax whose rows' sums are known.  S = Q K^T with the keys as columns, so that a column's entries lie in two lanes' registers and
// nothing is exchanged before the end; every sum belongs to one wave, in a fixed order.
//
// A wave keeps its keys as operands in registers for the whole call and the rows come by, 32 at a time, through LDS.
//
// What bounds it: the vector instructions (an fma, an exponential and an addition a score), the products and the reads of their operands from LDS, which
// hide each other in part: 2048 tokens of 32 heads over 32768 keys take 537 to 553 us by box, 0.97 to 1.0 PFLOP/s, without the vector work 407, without loads of
// rows as well 382, the products alone as a probe has them 279.  Without a tile's exponentials beside the next one's products 560; a tile that
// waits for the next step's 589; a row a lane, so that a tile has one lse a lane, 575; eight waves a workgroup 558; 128 keys and one wave a SIMD 895.
#include "paged.h"

#include <math.h>
#include <type_traits>

namespace kvs {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kRows = 32;               // rows of a tile
template <int ROW_B> constexpr int kStepRows = ROW_B <= 256 ? 128 : 64;           // rows between two barriers
constexpr int kPieceRows = 64;          // rows that pieces are counted in
constexpr int kMaxPieces = 16;
// Launches of fewer workgroups than fill the chip cut their rows, into four times as many.  (Of fewer than 1024, 8 contexts of 4000 with 48 tokens of 28 heads
// each 33 -> 45 us; into twice as many, 6000 tokens of 6000 264 -> 272.)
constexpr int64_t kCutBelow = 512;
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
    constexpr int RPL = kWave / CPR;                         // rows a load moves
    constexpr int kStep = kStepRows<ROW_B>, kStepsInfo = kThreads / kStep;
    constexpr int NQ = kStep / RPL / kWaves;                 // loads of a wave for a step's rows
    constexpr int NT = kStep / kRows;                        // tiles of a step
    __shared__ __attribute__((aligned(16))) char q_s[2][kStep * ROW_B];
    __shared__ __attribute__((aligned(16))) float lse_s[2][kThreads];       // of a workgroup's number of rows
    __shared__ __attribute__((aligned(16))) int pos_s[2][kThreads];
    __shared__ int span_s[2][kWaves][3];                     // of 64 rows: lowest position, highest, lowest of those that see anything

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hf = lane >> 5, ln = lane & 31;
    const int g = (int)(blockIdx.x % (uint32_t)n_kv_heads);
    int rest = (int)(blockIdx.x / (uint32_t)n_kv_heads);
    const int kb = rest % key_blocks;
    rest /= key_blocks;
    const int piece = rest % pieces, b = rest / pieces;
    const int end = end_of(pg, b), len = min(end, pg.max_ctx);
    const int wg_lo = kb * kWgKeys<DTYPE>;
    if (wg_lo >= len) return;
    const int my_lo = wg_lo + wave * NB * 32, my_hi = min(my_lo + NB * 32, len) - 1;   // the wave's keys
    int tok0, n_tok;
    tokens_of(pg, b, tok0, n_tok);
    const int grp = n_q_heads / n_kv_heads;
    const int rows = n_tok * grp;
    const int steps = (rows + kStep - 1) / kStep, per_piece = (steps + pieces - 1) / pieces;
    const int st_lo = min(piece * per_piece, steps), st_hi = min(st_lo + per_piece, steps);

    // ---- keys ---------------------------------------------------------------------------------------------------
    u32x4_t kreg[NB][NS];
    bool there[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int key = my_lo + nb * 32 + ln;
        const int at = granule_of(pg, b, key / kGranule);
        there[nb] = at >= 0 && key < len;
        const char *from = k_pool + (((int64_t)max(at, 0) * kGranule + key % kGranule) * n_kv_heads + g) * ROW_B;
#pragma unroll
        for (int c = 0; c < NS; ++c) kreg[nb][c] = *reinterpret_cast<const u32x4_t *>(from + (2 * c + hf) * 16);
    }

    // ---- rows ---------------------------------------------------------------------------------------------------
    auto swz = [](int r) { return CPR >= 16 ? (r & 15) : (r & 7); };
    // Rows go from memory straight into LDS, 16 bytes a lane; chunk c of row r lies at c ^ swz(r).  A step is the same number of bytes
    // further on for every lane where the query heads of a KV head divide 64; else its lanes follow their rows by additions.
    // (By hand: the compiler would wait for all loads in flight before every LDS read.)
    const int dh = kStep % grp, info_dt = kThreads / grp, info_dh = kThreads % grp;
    const int64_t stride = (int64_t)n_q_heads * ROW_B, inc = (int64_t)(kStep / grp) * stride;
    const int wrap = (n_q_heads - grp) * ROW_B;
    const char *q_base = q_new + ((int64_t)tok0 * n_q_heads + g * grp) * ROW_B + st_lo * inc;
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&q_s[0][0]);
    struct Row { int t, h; };
    auto row_at = [&](int r) { return Row{r / grp, r % grp}; };
    Row info = row_at(st_lo * kStep + tid);
    int64_t q_off[NQ];                                       // from q_base
    int q_head[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        const int r = (j * kWaves + wave) * RPL + lane / CPR;
        const Row at = row_at(st_lo * kStep + r);
        q_off[j] = at.t * stride - st_lo * inc + at.h * ROW_B + ((lane % CPR) ^ swz(r)) * 16;
        q_head[j] = at.h;
    }
    float lse_next = 0.f;
    int pos_next = -1;
    auto stage = [&](int st) {
        const uint32_t dst = lds_base + (uint32_t)(((st - st_lo) & 1) * (kStep * ROW_B) + wave * 1024);
        if (dh == 0 && (st + 1) * kStep <= rows) {
#pragma unroll
            for (int j = 0; j < NQ; ++j)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst + j * (kWaves * 1024)), "v"((uint32_t)q_off[j]), "s"(q_base) : "memory");
        } else {
#pragma unroll
            for (int j = 0; j < NQ; ++j) {
                const int r = st * kStep + (j * kWaves + wave) * RPL + lane / CPR;
                const char *from = r < rows ? q_base + q_off[j] : q_new;     // (rows behind the last: any)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(dst + j * (kWaves * 1024)), "v"(from) : "memory");
                q_head[j] += dh;
                const bool over = q_head[j] >= grp;
                q_head[j] -= over ? grp : 0;
                q_off[j] += dh * ROW_B + (over ? wrap : 0);
            }
        }
        q_base += inc;
    };
    auto fetch_info = [&]() {
        pos_next = -1;
        lse_next = 0.f;
        if (info.t < n_tok) {
            lse_next = lse[(int64_t)(tok0 + info.t) * n_q_heads + g * grp + info.h] * 1.4426950408889634f;
            pos_next = position_of(pg, tok0, n_tok, info.t, len, end);
            if (lse_next == -INFINITY) pos_next = -1;        // saw nothing
        }
        info.t += info_dt;
        info.h += info_dh;
        if (info.h >= grp) { info.h -= grp; ++info.t; }
    };
    const int window = pg.window, n_first = window ? pg.n_first : 0;
    float acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[nb] = 0.f;
    if (st_lo < st_hi) { fetch_info(); stage(st_lo); }
    for (int st = st_lo; st < st_hi; ++st) {
        const int buf = (st - st_lo) & 1, sub = (st - st_lo) % kStepsInfo, ibuf = ((st - st_lo) / kStepsInfo) & 1;
        if (sub == 0) {
            int lo = pos_next, hi = pos_next, low = pos_next < 0 ? 0x7fffffff : pos_next;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                lo = min(lo, __shfl_xor(lo, o));
                hi = max(hi, __shfl_xor(hi, o));
                low = min(low, __shfl_xor(low, o));
            }
            lse_s[ibuf][tid] = lse_next;
            pos_s[ibuf][tid] = pos_next;
            if (lane == 0) { span_s[ibuf][wave][0] = lo; span_s[ibuf][wave][1] = hi; span_s[ibuf][wave][2] = low; }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the step's rows have landed
        __syncthreads();
        if (st + 1 < st_hi) {
            stage(st + 1);
            if (sub == kStepsInfo - 1) fetch_info();
        }
        constexpr int WPS = kStep / kWave;                   // waves that looked at a step's rows
        int pmin = 0x7fffffff, pmax = -1, plow = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < WPS; ++i) {
            pmin = min(pmin, span_s[ibuf][sub * WPS + i][0]);
            pmax = max(pmax, span_s[ibuf][sub * WPS + i][1]);
            plow = min(plow, span_s[ibuf][sub * WPS + i][2]);
        }
        pmin = __builtin_amdgcn_readfirstlane(pmin);
        pmax = __builtin_amdgcn_readfirstlane(pmax);
        plow = __builtin_amdgcn_readfirstlane(plow);
        if (pmax < my_lo || (window && my_hi <= plow - window && my_lo >= n_first)) continue;
        const bool masked = my_hi > pmin || (window && my_lo <= pmax - window && my_hi >= n_first);
        auto scores = [&](int t, floatx16 (&s)[NB]) {
            const int r = t * kRows + ln;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[nb][i] = 0.f;
#pragma unroll
            for (int c = 0; c < NS; ++c) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t *>(q_s[buf] + r * ROW_B + ((2 * c + hf) ^ swz(r)) * 16);
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
        };
        auto add_up = [&](int t, const floatx16 (&s)[NB], auto with_mask) {
            const int r0 = sub * kStep + t * kRows + 4 * hf;
            float sum[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) sum[nb] = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {                    // entry 4 q + u is row 8 q + 4 hf + u
                const float4 l4 = *reinterpret_cast<const float4 *>(&lse_s[ibuf][r0 + 8 * q]);
                const float l[4] = {l4.x, l4.y, l4.z, l4.w};
                int p[4] = {};
                if constexpr (decltype(with_mask)::value) {
                    const int4 p4 = *reinterpret_cast<const int4 *>(&pos_s[ibuf][r0 + 8 * q]);
                    p[0] = p4.x; p[1] = p4.y; p[2] = p4.z; p[3] = p4.w;
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float e[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) e[u] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][4 * q + u], scale_log2, -l[u]));
                    if constexpr (decltype(with_mask)::value) {
                        const int key = my_lo + nb * 32 + ln;
#pragma unroll
                        for (int u = 0; u < 4; ++u) e[u] = key <= p[u] && (!window || key > p[u] - window || key < n_first) ? e[u] : 0.f;
                    }
                    sum[nb] += (e[0] + e[1]) + (e[2] + e[3]);
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[nb] += sum[nb];
        };
        // Products of tile t beside the exponentials of the tile before, whose rows' lse begin at l_at.  A slice is the products of 32 (fp32: 8) of a
        // row's channels and as large a part of the exponentials; the fences keep it together, and operands are read two slices ahead.
        // (2048 tokens of 32 heads over 32768 keys 560 -> 537 us; one slice ahead 550; four 537.)
        constexpr int AH = 2;
        auto read_q = [&](int at) { return *reinterpret_cast<const u32x4_t *>(q_s[buf] + (at / NS * kRows + ln) * ROW_B + ((2 * (at % NS) + hf) ^ swz(ln)) * 16); };
        auto both = [&](int t, floatx16 (&s)[NB], const floatx16 (&before)[NB], const float *l_at, u32x4_t (&w)[AH], auto exps) __attribute__((always_inline)) {
            constexpr bool EXPS = decltype(exps)::value;
            constexpr int EACH = 16 * NB / NS, SLICES = 4 * NB / EACH > 0 ? 4 * NB / EACH : 1;
            const floatx16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            float4 l4 = {}, l4_n = {};
            if (EXPS) l4 = *reinterpret_cast<const float4 *>(l_at);
            float sum[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) sum[nb] = 0.f;
#pragma unroll
            for (int c = 0; c < NS; ++c) {
                const u32x4_t w_n = read_q(min(t * NS + c + AH, NT * NS - 1));
                if (EXPS && c % SLICES == 0 && c / SLICES < 3) l4_n = *reinterpret_cast<const float4 *>(l_at + 8 * (c / SLICES + 1));
                const float l[4] = {l4.x, l4.y, l4.z, l4.w};
                float e[EACH];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (F32) {
#pragma unroll
                        for (int u = 0; u < 4; ++u) s[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[(t * NS + c) % AH][u]), __uint_as_float(kreg[nb][c][u]), c + u == 0 ? zero : s[nb], 0, 0, 0);
                    } else {
                        s[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w[(t * NS + c) % AH]), as_bf16x8(kreg[nb][c]), c == 0 ? zero : s[nb], 0, 0, 0);
                    }
                    if (EXPS && nb == 0) {
#pragma unroll
                        for (int u = 0; u < EACH; ++u) {
                            const int at = c * EACH + u;
                            e[u] = __builtin_amdgcn_exp2f(__builtin_fmaf(before[at / 4 % NB][at / (4 * NB) * 4 + at % 4], scale_log2, -l[at % 4]));
                        }
                    }
                }
                if (EXPS) {
#pragma unroll
                    for (int u = 0; u < EACH; ++u) sum[(c * EACH + u) / 4 % NB] += e[u];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) asm volatile("" : "+v"(sum[nb]));
                }
                w[(t * NS + c) % AH] = w_n;
                if (EXPS && c % SLICES == SLICES - 1) l4 = l4_n;
                __builtin_amdgcn_sched_barrier(0);
            }
            if (EXPS) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[nb] += sum[nb];
            }
        };
        if (masked || (st + 1) * kStep > rows) {
#pragma unroll 1
            for (int t = 0; t < NT && st * kStep + t * kRows < rows; ++t) {
                const int *const span = span_s[ibuf][sub * WPS + t * kRows / kWave];
                if (__builtin_amdgcn_readfirstlane(span[1]) < my_lo) continue;
                floatx16 s[NB];
                scores(t, s);
                if (window || my_hi > __builtin_amdgcn_readfirstlane(span[0])) add_up(t, s, std::true_type{});
                else add_up(t, s, std::false_type{});
            }
        } else {
            const float *const l_at = &lse_s[ibuf][sub * kStep + 4 * hf];
            floatx16 s[2][NB];
            u32x4_t w[AH];
#pragma unroll
            for (int i = 0; i < AH; ++i) w[i] = read_q(i);
            both(0, s[0], s[1], l_at, w, std::false_type{});
#pragma unroll
            for (int t = 1; t < NT; ++t) both(t, s[t & 1], s[(t - 1) & 1], l_at + (t - 1) * kRows, w, std::true_type{});
            add_up(NT - 1, s[(NT - 1) & 1], std::false_type{});
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float total = acc[nb] + __shfl_xor(acc[nb], 32);
        const int key = my_lo + nb * 32 + ln;
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

// Few rows a request, a decode step's: the cache's bytes bound it, half of what the attention itself reads.  A wave holds the rows as
// operands and takes every fourth tile of 32 keys of the workgroup's piece, two of them on their way into LDS slots of its own
// (global to LDS, 16 bytes a lane, no registers, no barrier).  Sums of kFlush tiles wait in LDS until they are added to the
// mass that was: loads and stores of its own in every tile would have to be waited for in order with the keys.
// Requests of more than 32 rows, which the host cannot see, come here too where there are few on average: block by block.
constexpr int kFlush = 16;

template <int DTYPE, int D>
__global__ __launch_bounds__(kThreads, 2) void mass_few_kernel(
    const Paged pg, int n_q_heads, int n_kv_heads, int pieces, int piece_tiles, const char *__restrict__ k_pool, const char *__restrict__ q_new,
    const float *__restrict__ lse, float scale_log2, float decay, const float *mass, float *mass_out, int64_t mass_stride)
{
    constexpr bool F32 = DTYPE == KVS_F32;
    constexpr int ROW_B = D * (F32 ? 4 : 2);
    constexpr int CPR = ROW_B / 16;
    constexpr int NS = CPR / 2;
    constexpr int RPL = kWave / CPR;                         // rows a load moves
    constexpr int NH = kGranule / RPL, NL = 2 * NH;          // loads of half a tile, of a tile
    constexpr int TILE_B = 32 * ROW_B;
    extern __shared__ __attribute__((aligned(16))) char lds[];       // two slots a wave
    __shared__ float sum_s[kWaves][kFlush][32];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hf = lane >> 5, ln = lane & 31;
    const int g = (int)(blockIdx.x % (uint32_t)n_kv_heads);
    const int rest = (int)(blockIdx.x / (uint32_t)n_kv_heads);
    const int b = rest % pg.batch, piece = rest / pg.batch;
    const int end = end_of(pg, b), len = min(end, pg.max_ctx);
    const int tiles = (len + 31) / 32;
    const int p_lo = (int)min((int64_t)piece * piece_tiles, (int64_t)tiles), p_hi = (int)min((int64_t)p_lo + piece_tiles, (int64_t)tiles);
    if (p_lo >= p_hi) return;
    int tok0, n_tok;
    tokens_of(pg, b, tok0, n_tok);
    const int grp = n_q_heads / n_kv_heads, rows = n_tok * grp;
    const int window = pg.window, n_first = window ? pg.n_first : 0;
    const int64_t out_at = ((int64_t)b * n_kv_heads + g) * mass_stride;

    char *const my_lds = lds + wave * (2 * TILE_B);
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)my_lds);
    const uint32_t row_bytes = (uint32_t)n_kv_heads * ROW_B;
    auto swz = [](int r) { return CPR >= 16 ? (r & 15) : (r & 7); };
    uint32_t k_off[NH];
#pragma unroll
    for (int j = 0; j < NH; ++j) {
        const int r = j * RPL + lane / CPR;
        k_off[j] = (uint32_t)r * row_bytes + (uint32_t)((lane % CPR) ^ swz(r)) * 16u;
    }
    // By hand, as in attention_paged.hip: the compiler would wait for all loads in flight before every LDS read.  Keys are read once, and the loads
    // say so (64 contexts of 4096 to 16384 281 -> 259 us).
    auto load_1k = [&](uint32_t dst, uint32_t off, const char *base) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(dst), "v"(off), "s"(base) : "memory");
    };
    const uint64_t granule_bytes = (uint64_t)row_bytes * kGranule;

    const int blocks = max(1, (rows + 31) / 32);             // no rows: everything decays
    for (int blk = 0; blk < blocks; ++blk) {
        // ---- rows ---------------------------------------------------------------------------------------------------
        const int rq = blk * 32 + ln;
        const int t_own = rows ? min(rq, rows - 1) / grp : 0, h_own = rows ? min(rq, rows - 1) - t_own * grp : 0;
        int pos = -1;
        float lse2 = 0.f;
        u32x4_t qreg[NS];
#pragma unroll
        for (int c = 0; c < NS; ++c) qreg[c] = u32x4_t{0u, 0u, 0u, 0u};
        if (rows) {
            const int64_t row = (int64_t)(tok0 + t_own) * n_q_heads + g * grp + h_own;
            pos = rq < rows ? position_of(pg, tok0, n_tok, t_own, len, end) : -1;
            lse2 = lse[row] * 1.4426950408889634f;
            if (lse2 == -INFINITY) pos = -1;                 // saw nothing
#pragma unroll
            for (int c = 0; c < NS; ++c) qreg[c] = *reinterpret_cast<const u32x4_t *>(q_new + row * ROW_B + (2 * c + hf) * 16);
        }
        int pmin = pos, pmax = pos, plow = pos < 0 ? 0x7fffffff : pos;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            pmin = min(pmin, __shfl_xor(pmin, o));
            pmax = max(pmax, __shfl_xor(pmax, o));
            plow = min(plow, __shfl_xor(plow, o));
        }
        pmin = __builtin_amdgcn_readfirstlane(pmin);
        pmax = __builtin_amdgcn_readfirstlane(pmax);
        plow = __builtin_amdgcn_readfirstlane(plow);
        float l_of[16];                                      // entry r of a product is row 8 (r >> 2) + 4 hf + (r & 3)
        int p_of[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            l_of[r] = __shfl(lse2, 8 * (r >> 2) + 4 * hf + (r & 3));
            p_of[r] = __shfl(pos, 8 * (r >> 2) + 4 * hf + (r & 3));
        }
        // ---- the piece's tiles that any of them sees: [p_lo, head) and [low, high) ---------------------------------
        int low = window && pmax >= 0 ? max(plow - window + 1, 0) / 32 : 0;
        int head = min(low, (int)(((int64_t)n_first + 31) / 32));
        const int high = min(p_hi, pmax < 0 ? 0 : pmax / 32 + 1);
        low = max(low, p_lo);
        head = max(min(head, high), p_lo);
        const int total = head - p_lo + max(high - low, 0);
        const int mine = max(0, (total - wave + kWaves - 1) / kWaves);
        auto tile_of = [&](int i) { const int t = p_lo + wave + kWaves * i; return t < head ? t : t - head + low; };
        int place = -1;
        auto look_up = [&](int i0) {
            const int i = i0 + (lane >> 1);
            place = i < mine ? granule_of(pg, b, 2 * tile_of(i) + (lane & 1)) : -1;
        };
        auto stage = [&](int i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = max(__builtin_amdgcn_readlane(place, 2 * (i & 31) + h), 0);
                const char *base = k_pool + (uint64_t)(uint32_t)at * granule_bytes + (uint32_t)g * ROW_B;
#pragma unroll
                for (int j = 0; j < NH; ++j) load_1k(lds_base + (uint32_t)((i & 1) * TILE_B + (h * NH + j) * 1024), k_off[j], base);
            }
        };
        // what becomes of a key: in the first block its mass decays
        auto store = [&](int key, float sum) {
            if (key >= len) return;
            const float old = blk ? mass_out[out_at + key] : mass ? mass[out_at + key] : 0.f;
            mass_out[out_at + key] = blk ? old + sum : __builtin_fmaf(decay, old, sum);
        };
        auto flush = [&](int i0, int n) {                    // the sums of tiles i0 .. i0 + n - 1
            for (int e = lane; e < n * 32; e += kWave) store(tile_of(i0 + e / 32) * 32 + e % 32, sum_s[wave][e / 32][e % 32]);
        };
        look_up(0);
        if (mine > 0) stage(0);
        if (mine > 1) stage(1);
        int none_at = place;                                 // of the tiles that are worked on
        for (int i = 0; i < mine; ++i) {
            const int x0 = tile_of(i) * 32;
            if ((i & 31) == 0) none_at = place;
            const bool none[2] = {__builtin_amdgcn_readlane(none_at, 2 * (i & 31)) < 0, __builtin_amdgcn_readlane(none_at, 2 * (i & 31) + 1) < 0};
            if (((i + 2) & 31) == 0 && i + 2 < mine) look_up(i + 2);
            if (i + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NL) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const char *const kt = my_lds + (i & 1) * TILE_B;
            floatx16 s;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
            for (int c = 0; c < NS; ++c) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t *>(kt + ln * ROW_B + ((2 * c + hf) ^ swz(ln)) * 16);
                if constexpr (F32) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(qreg[c][u]), __uint_as_float(w[u]), s, 0, 0, 0);
                } else {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(qreg[c]), as_bf16x8(w), s, 0, 0, 0);
                }
            }
            if (i + 2 < mine) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // what lay in the slot has been read
                stage(i + 2);
            }
            const int key = x0 + ln;
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool seen = key <= p_of[r] && (!window || key > p_of[r] - window || key < n_first);
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], scale_log2, -l_of[r]));
                sum += seen ? e : 0.f;
            }
            sum += __shfl_xor(sum, 32);
            if (hf == 0) sum_s[wave][i % kFlush][ln] = none[ln >> 4] ? 0.f : sum;
            if (i % kFlush == kFlush - 1) flush(i + 1 - kFlush, kFlush);
        }
        flush(mine - mine % kFlush, mine % kFlush);
        // ---- and those that none sees -------------------------------------------------------------------------------
        if (blk == 0 && !(mass == mass_out && decay == 1.f)) {
            const int gap_lo = head, gap_hi = max(low, head);              // tiles of the piece between the two ranges, and behind them
            for (int key = max(gap_lo, p_lo) * 32 + tid; key < min(gap_hi, p_hi) * 32; key += kThreads) store(key, 0.f);
            for (int key = max(max(high, gap_hi), p_lo) * 32 + tid; key < p_hi * 32; key += kThreads) store(key, 0.f);
        }
        if (blk + 1 < blocks) __syncthreads();               // (the next rows' tiles may fall to other waves)
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
    const int64_t steps = n_new * (shape->n_q_heads / shape->n_kv_heads) / (batch * kPieceRows);
    if (wgs <= 0 || wgs >= kCutBelow || batch * shape->n_kv_heads > 65535) return 1;
    int64_t p = (4 * kCutBelow + wgs - 1) / wgs;
    if (p > (steps + 3) / 4) p = (steps + 3) / 4;
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

template <int DTYPE, int D>
kvs_status launch_few(const kvs_shape *shape, const kvs_paged_cache *c, const Paged &pg, const void *q, const float *lse, float scale, float decay, const float *mass, float *mass_out,
                      int64_t mass_stride, hipStream_t hs)
{
    static DeviceOnce once;
    constexpr int lds = kWaves * 2 * 32 * D * (DTYPE == KVS_F32 ? 4 : 2);
    kvs_status st = once_per_device(once, [&]() -> kvs_status {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&mass_few_kernel<DTYPE, D>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        return e == hipSuccess ? KVS_OK : fail(KVS_EHIP, "kvs_mass_paged: %s", hipGetErrorString(e));
    });
    if (st != KVS_OK) return st;
    const int64_t units = (int64_t)pg.batch * shape->n_kv_heads, tiles = (pg.max_ctx + 31) / 32;
    // One workgroup for each place on the chip, and none of more than 128 tiles.  (512, 1024, 2048 workgroups, us: 8 contexts of 2000 to 8000 of
    // 8 heads 22.2, 23.1, 24.3; 4 of 10000 to 40000 of 4 30.8, 32.9, 34.8; 64 of 100 to 400 of 8 13.2, 15.2, 15.3; 64 of 4096 to 16384, before loads said that keys
    // are read once, 280 each (now 258 to 266), 313 with pieces as long as they come.)
    int64_t pieces = (512 + units - 1) / units;
    if (pieces < (tiles + 127) / 128) pieces = (tiles + 127) / 128;
    int64_t piece_tiles = (tiles + pieces - 1) / pieces;
    piece_tiles = piece_tiles < 2 * kWaves ? 2 * kWaves : (piece_tiles + kWaves - 1) / kWaves * kWaves;
    pieces = (tiles + piece_tiles - 1) / piece_tiles;
    if (pieces * units > kMostWgs) return fail(KVS_EINVAL, "kvs_mass_paged: too many rows in one call");
    hipLaunchKernelGGL((mass_few_kernel<DTYPE, D>), dim3((unsigned)(pieces * units)), dim3(kThreads), lds, hs, pg, shape->n_q_heads, shape->n_kv_heads, (int)pieces, (int)piece_tiles,
                       (const char *)c->k, (const char *)q, lse, scale * 1.4426950408889634f, decay, mass, mass_out, mass_stride);
    return check_launch("kvs_mass_paged");
}

// Whether a call's rows are so few that the keys' bytes bound it.
inline bool few_rows(const kvs_shape *shape, int64_t batch, int64_t n_new) { return n_new * (shape->n_q_heads / shape->n_kv_heads) <= 32 * batch; }

} // namespace

size_t mass_paged_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t max_ctx, int64_t n_new)
{
    if (check_shape(shape) != KVS_OK || batch <= 0 || max_ctx <= 0 || n_new <= 0) return 256;
    if (few_rows(shape, batch, n_new)) return 256;
    // no more than kMaxPieces pieces, and of kWgKeys keys fewer than 4 kCutBelow and what one more piece makes
    const int64_t all = (int64_t)batch * shape->n_kv_heads * max_ctx, most = (int64_t)5 * kCutBelow * kWgKeys<KVS_BF16>;
    return ((size_t)(all < most / kMaxPieces ? all * kMaxPieces : most) * 4 + 255) / 256 * 256;
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
    if (!isfinite(scale * 1.4426950408889634f)) return fail(KVS_EINVAL, "%s: a scale of %g", me, (double)scale);
    if (!isfinite(decay) || decay < 0.f) return fail(KVS_EINVAL, "%s: a decay of %g", me, (double)decay);
    if (mass_stride < pages->max_ctx) return fail(KVS_EINVAL, "%s: a mass stride of %lld for contexts of up to %lld", me, (long long)mass_stride, (long long)pages->max_ctx);
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(KVS_EINVAL, "%s: workspace must be 256-byte aligned", me);
    if (!workspace) workspace_bytes = 0;
    if (pages->batch == 0 || pg.max_ctx == 0) return KVS_OK;
    if (!mass_out) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    const size_t mass_bytes = (size_t)pages->batch * shape->n_kv_heads * mass_stride * sizeof(float);
    if (mass && mass != mass_out && overlap(mass, mass_bytes, mass_out, mass_bytes)) return fail(KVS_EINVAL, "%s: mass_out overlaps mass without being it", me);
    if (n_new > 0 && (!q_new || !lse)) return fail(KVS_EINVAL, "%s: NULL tensor pointer", me);
    if (!aligned16(q_new)) return fail(KVS_EINVAL, "%s: Q must be 16-byte aligned", me);
    const size_t pool = pool_bytes(shape, cache), heads = (size_t)n_new * shape->n_q_heads, batch = (size_t)pages->batch;
    st = check_apart(me, {{mass_out, mass_bytes, "mass_out"}},
                     {{q_new, heads * shape->head_dim * elem_bytes(shape->dtype), "q_new"}, {lse, heads * sizeof(float), "lse"}, {cache->k, pool, "the cache's K"},
                      {cache->v, pool, "the cache's V"}, {pages->table, batch * pages->width * 4, "the page table"}, {pages->ctx_len, batch * 4, "ctx_len"},
                      {cu_new, (batch + 1) * 4, "cu_new"}, {sel_pos, (size_t)n_new * 4, "sel_pos"}});
    if (st != KVS_OK) return st;
    const bool wide = shape->head_dim == 128;
    hipStream_t hs = (hipStream_t)stream;
    if (few_rows(shape, pg.batch, n_new)) {
#define KVS_MF(DT, DD) launch_few<DT, DD>(shape, cache, pg, q_new, lse, scale, decay, mass, mass_out, mass_stride, hs)
        if (shape->dtype == KVS_F32) return wide ? KVS_MF(KVS_F32, 128) : KVS_MF(KVS_F32, 64);
        return wide ? KVS_MF(KVS_BF16, 128) : KVS_MF(KVS_BF16, 64);
#undef KVS_MF
    }
    const int64_t key_blocks = blocks_of(shape, pg.max_ctx);
    int pieces = pieces_of(shape, pg.batch, pg.max_ctx, n_new);
    const int64_t fit = (int64_t)(workspace_bytes / 4) / ((int64_t)pg.batch * shape->n_kv_heads * pg.max_ctx);
    if (pieces > fit) pieces = fit < 1 ? 1 : (int)fit;
    if (key_blocks * pieces * pg.batch * shape->n_kv_heads > kMostWgs) return fail(KVS_EINVAL, "%s: too many rows in one call", me);
#define KVS_MP(DT, DD) launch<DT, DD>(shape, cache, pg, key_blocks, pieces, q_new, lse, scale, decay, mass, mass_out, mass_stride, (float *)workspace, hs)
    if (shape->dtype == KVS_F32) return wide ? KVS_MP(KVS_F32, 128) : KVS_MP(KVS_F32, 64);
    return wide ? KVS_MP(KVS_BF16, 128) : KVS_MP(KVS_BF16, 64);
#undef KVS_MP
}
