// kvs_store_kv8: rows of K and V into a cache held in 8 bits with a scale for each block of tokens and KV head.
//
// A block's scale comes from the largest magnitude among the rows that it takes, so its rows are needed twice: once for
// that maximum and once to be divided by it.  They stay in registers in between, so memory sees them once: 2 or 4 bytes
// an element in, 1 byte out, plus the kept rows' codes where a block's scale grows.
//
// Rows in a row (no list): a workgroup has one block and its share of the units, a unit being one KV head of K or of V.  A wave
// holds up to 32 rows of a unit, so a unit takes a team of 1, 2 or 4 waves (`waves`), which meet in LDS for their maximum.
//
// A list: its entries of one block, and skipped ones between them, are a run.  A wave has a few entries of the list, finds the runs
// that begin there from one load of the positions, and takes 64 pieces of the rows of each, 4 heads of 256 bytes; no wave waits
// for another.  Skipped entries end no run: the wave of the last one before a stretch of them looks through it (0.9 us for 512
// entries; 1000 rows 8.0 us, with 3096 skipped entries behind them 10.8), and the wave that begins behind it looks back.  Which
// entry a row takes is settled in LDS: the highest that names it, whatever order the entries of a block come in.  A lane has the same
// piece of up to 8 rows: its maximum runs over the rows first, then over the lanes of its head (no exchange beyond 16 lanes), and the
// scale is made in every lane that needs it.  What a wave waits for is one trip to memory for the positions, one for the rows
// and old scales, and where a scale grows one or two for the codes that it rounds again, head by head with all lanes.  (4424 of 32768
// rows of 8 heads, blocks of 32: a workgroup for each entry 35.6 us, a chunk of the list and one unit a workgroup 25.8, a wave a run
// with whole heads one after the other 20, issue bound; this 13.6 in a trace, 13.0 in a full queue.  The first time over a filled
// cache, where 2 % of the scales grow, 18 to 21; where all grow 41, of which the codes' 134 MB would take 26 at a copy's rate.  One
// row in each of 64 blocks of 32 4.0, in blocks of 128 whose scales all grow 39: 128 rows of 8 heads, one head after the other.)
#include "cache8.h"

#include <math.h>

#include <type_traits>

namespace kvs {
namespace {

constexpr int kThreads = 256;
constexpr int kWaveRows = 32;
constexpr int kMaxBlock = 128;
constexpr int kListRows = 8;           // rows of a run that a lane holds
constexpr int kAgain = 2;              // 16-byte pieces of kept rows that a lane holds
constexpr int kMaxChunk = 32;          // entries in which a wave looks for runs; runs that go on behind them are followed
constexpr int kSkips = 8;              // times 64 entries asked for at once where a list is followed far (16: a wave a SIMD fewer, 4424 of 32768 rows 5 % slower)
constexpr int64_t kManyWaves = 16384;  // waves from which they get more entries each

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

// largest of a number's magnitude as bits: magnitudes order as whole numbers, NaN above infinity above the rest
template <int DTYPE>
__device__ __forceinline__ uint32_t magnitude_bits(const uint4 w)
{
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DTYPE == KVS_BF16) bits = max(bits, max((ww[j] << 16) & 0x7fffffffu, ww[j] & 0x7fff0000u));
        else bits = max(bits, ww[j] & 0x7fffffffu);
    }
    return bits;
}

// over each aligned group of LANES (8, 16, 32, 64) lanes
template <int LANES>
__device__ __forceinline__ uint32_t head_max_bits(uint32_t v)
{
    if constexpr (LANES == 8) {
        v = max(v, (uint32_t)__shfl_xor((int)v, 4));
        v = max(v, (uint32_t)__shfl_xor((int)v, 2));
        return max(v, (uint32_t)__shfl_xor((int)v, 1));
    }
    v = max(v, (uint32_t)dpp_i32<0x128>((int)v));
    v = max(v, (uint32_t)dpp_i32<0x124>((int)v));
    v = max(v, (uint32_t)dpp_i32<0x122>((int)v));
    v = max(v, (uint32_t)dpp_i32<0x121>((int)v));
    if constexpr (LANES >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    if constexpr (LANES >= 64) v = max(v, (uint32_t)__shfl_xor((int)v, 32));
    return v;
}

// what becomes of a block's scale, and how its rows are written
struct NewScale {
    float scale, inv, ratio;
    bool odd, again;          // a NaN or infinity is among the rows; kept rows have to be rounded again
};
template <int CODE>
__device__ __forceinline__ NewScale new_scale(uint32_t bits, float old, bool keeps)
{
    NewScale n;
    const float most = __uint_as_float(bits);
    n.odd = bits >= 0x7f800000u || (keeps && old != old);
    const float need = most > 0.f ? fmaxf(most * (1.f / top_code<CODE>()), kLeastScale) : 0.f;
    n.scale = n.odd ? __uint_as_float(0x7fc00000u) : keeps ? fmaxf(old, need) : need;
    n.inv = n.scale > 0.f ? 1.f / n.scale : 0.f;
    n.again = keeps && n.scale > 0.f && n.scale != old;
    n.ratio = n.again ? old / n.scale : 1.f;
    return n;
}

// the codes of a 16-byte piece (codes of 0 under a scale that is no number)
template <int DTYPE, int CODE>
__device__ __forceinline__ void write_codes(uint8_t *dst, const uint4 w, float by, bool odd)
{
    if constexpr (DTYPE == KVS_BF16) {
        uint2 c;
        c.x = nearest_codes<CODE>(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), by);
        c.y = nearest_codes<CODE>(bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w), by);
        *reinterpret_cast<uint2 *>(dst) = odd ? make_uint2(0u, 0u) : c;
    } else {
        const uint32_t c = nearest_codes<CODE>(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w), by);
        *reinterpret_cast<uint32_t *>(dst) = odd ? 0u : c;
    }
}

// four codes in steps of a scale that is 1 / ratio times theirs
template <int CODE>
__device__ __forceinline__ uint32_t again4(uint32_t codes, float ratio)
{
    float x[4];
    widen_codes<CODE>(CODE == KVS_E4M3 ? numbers_only(codes) : codes, x);
    return nearest_codes<CODE>(x[0], x[1], x[2], x[3], ratio);
}

// Kept rows stand for what they stood for, in steps of the new scale: `rows` of them from `to` on, those with src < 0.
template <int CODE, int D>
__device__ __forceinline__ void round_again(uint8_t *to, int64_t row_bytes, int rows, const int *src, float ratio, int lane)
{
    constexpr int CP = D / 16, N = kWaveRows * CP / kWave;    // 16-byte pieces of a row; of 32 rows, a lane's
    uint4 held[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + i * kWave, r = e / CP;
        held[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows && src[r] < 0) held[i] = reinterpret_cast<const uint4 *>(to + r * row_bytes)[e % CP];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane + i * kWave, r = e / CP;
        if (r >= rows || src[r] >= 0) continue;
        reinterpret_cast<uint4 *>(to + r * row_bytes)[e % CP] =
            make_uint4(again4<CODE>(held[i].x, ratio), again4<CODE>(held[i].y, ratio), again4<CODE>(held[i].z, ratio), again4<CODE>(held[i].w, ratio));
    }
}

// ---- rows row0 .. row0 + n_sel - 1 ---------------------------------------------------------------------------------
template <int DTYPE, int CODE, int D>
__global__ __launch_bounds__(kThreads) void store_rows_kernel(const StoreArgs a)
{
    constexpr int E = DTYPE == KVS_BF16 ? 8 : 4;           // elements of a 16-byte piece
    constexpr int PPR = D / E;                             // pieces of a row
    constexpr int RPI = kWave / PPR;                       // rows a wave loads at once
    constexpr int N = kWaveRows / RPI;                     // pieces a lane holds
    __shared__ int src_s[4][kWaveRows];                    // entry that a row of the wave's part takes, -1: the row is kept
    __shared__ uint32_t most_s[2][4];
    __shared__ float old_s[2][4];
    __shared__ int keeps_s[4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = 1 << a.block_log2, hk = a.n_kv_heads, units = 2 * hk;
    const int n_teams = 4 / a.waves, team = wave / a.waves, part = wave % a.waves, first_row = part * kWaveRows;
    const int64_t blk = (a.row0 >> a.block_log2) + blockIdx.x, block0 = blk << a.block_log2;

    if (blockIdx.y == 0) {
        for (int e = tid; e < block * (hk + 1); e += kThreads) {
            const int64_t r = block0 + (e & (block - 1));
            const int g = e >> a.block_log2;
            if (r < a.row0 || r >= a.row0 + a.n_sel) continue;
            if (g < hk) { if (a.dev_v) a.dev_v[(int64_t)g * a.n_rows + r] = 0.f; }
            else if (a.reused) a.reused[r] = 0;
        }
    }
    int *const src = src_s[wave];
    const int rows_here = (int)min((int64_t)block, a.n_rows - block0) - first_row;         // from the wave's first row on
    int mine = 0;
    if (lane < kWaveRows) {
        const int64_t e = block0 + first_row + lane - a.row0;
        mine = first_row + lane < block && e >= 0 && e < a.n_sel ? (int)e : -1;
        src[lane] = mine;
    }
    const bool keeps_part = __ballot(lane < kWaveRows && lane < rows_here && mine < 0) != 0;
    if (lane == 0) keeps_s[wave] = keeps_part;
    __syncthreads();
    bool keeps = false;
    for (int i = 0; i < a.waves; ++i) keeps |= keeps_s[team * a.waves + i] != 0;

    const int u_lo = (int)blockIdx.y * a.units_per_wg, n_units = min(a.units_per_wg, units - u_lo);
    int parity = 0;
    for (int k0 = 0; k0 < n_units; k0 += n_teams, parity ^= 1) {
        const bool live = k0 + team < n_units;
        const int u = u_lo + (live ? k0 + team : 0);
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
                const int e = src[i * RPI + sub];
                w[i] = make_uint4(0u, 0u, 0u, 0u);
                if (e >= 0) w[i] = stream_load16(from + ((int64_t)e * hk + g) * PPR + piece);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) bits = max(bits, magnitude_bits<DTYPE>(w[i]));
        }
        bits = head_max_bits<kWave>(bits);
        if (a.waves > 1) {
            // the old scale is read by the wave that will write the new one, and has arrived before the barrier; two sets in
            // turn: a wave writes to one again only behind the barrier of the round in between
            if (lane == 0) { most_s[parity][wave] = bits; old_s[parity][wave] = old; }
            __syncthreads();
            for (int i = 0; i < a.waves; ++i) bits = max(bits, most_s[parity][team * a.waves + i]);
            old = old_s[parity][team * a.waves];
        }
        if (!live) continue;
        const NewScale n = new_scale<CODE>(bits, old, keeps);
        const int64_t row_bytes = (int64_t)hk * D;
        uint8_t *to = (is_v ? a.v : a.k) + ((block0 + first_row) * hk + g) * D;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = i * RPI + sub;
            if (src[r] >= 0) write_codes<DTYPE, CODE>(to + r * row_bytes + piece * E, w[i], n.inv, n.odd);
        }
        if (n.again) round_again<CODE, D>(to, row_bytes, rows_here, src, n.ratio, lane);
        if (lane == 0 && part == 0) *scale_at = n.scale;
    }
}

// ---- the rows of a list --------------------------------------------------------------------------------------------
template <int DTYPE, int CODE, int D>
__global__ __launch_bounds__(kThreads) void store_list_kernel(const StoreArgs a)
{
    constexpr int E = DTYPE == KVS_BF16 ? 8 : 4, PPR = D / E;
    __shared__ int src_s[4][kMaxBlock];                    // entry that a row of the block takes, -1: the row is kept
    __shared__ int row_s[4][kMaxBlock];                    // the rows that take one, in order
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hk = a.n_kv_heads, pieces = hk * PPR, columns = (pieces + kWave - 1) / kWave;
    const bool is_v = (int)blockIdx.y >= columns;
    const int piece = ((int)blockIdx.y - (is_v ? columns : 0)) * kWave + lane;      // of a row, the lane's
    const bool inside = piece < pieces;
    const int g = piece / PPR;                             // its KV head
    int *const src = src_s[wave], *const row_at = row_s[wave];

    // lane i holds entry chunk0 + i: its block (-1: skipped, outside the cache), and whether a run begins there
    const int64_t chunk0 = ((int64_t)blockIdx.x * 4 + wave) * a.chunk;
    if (chunk0 >= a.n_sel) return;
    auto blk_of = [&](int p) -> int { return p >= 0 && p < a.n_rows ? p >> a.block_log2 : -1; };
    const int my_pos = chunk0 + lane < a.n_sel ? a.sel_pos[chunk0 + lane] : -1;
    int before = __builtin_amdgcn_readfirstlane(blk_of(chunk0 > 0 ? a.sel_pos[chunk0 - 1] : -1));
    const int my_blk = blk_of(my_pos);
    const uint64_t taken = __ballot(my_blk >= 0), own = ((uint64_t)1 << a.chunk) - 1;
    // Skipped entries end no run: what counts is the block of the last entry before that is not one.
    for (int64_t s = chunk0 - 1; (taken & own) && before < 0 && s > 0; s -= kSkips * kWave) {
        const int32_t *const at = a.sel_pos + (s - kWave);         // (before the list's begin where nothing is read)
        const int there = (int)min(s, (int64_t)(kSkips * kWave));
        int p[kSkips];
#pragma unroll
        for (int j = 0; j < kSkips; ++j) p[j] = j * kWave + 63 - lane < there ? at[lane - j * kWave] : -1;
#pragma unroll
        for (int j = 0; j < kSkips; ++j) {
            const uint64_t some = __ballot(blk_of(p[j]) >= 0);
            if (some && before < 0) before = __builtin_amdgcn_readlane(blk_of(p[j]), 63 - __builtin_clzll(some));
        }
    }
    const uint64_t left_of = taken & (((uint64_t)1 << lane) - 1);
    const int left_blk = __shfl(my_blk, left_of ? 63 - __builtin_clzll(left_of) : 0), left = left_of ? left_blk : before;
    const uint64_t begins = __ballot(my_blk >= 0 && my_blk != left);
    uint64_t runs = begins & own;
    if (blockIdx.y == 0 && my_blk >= 0 && lane < a.chunk) {
        if (a.reused) a.reused[my_pos] = 0;
        if (a.dev_v) for (int g = 0; g < hk; ++g) a.dev_v[(int64_t)g * a.n_rows + my_pos] = 0.f;
    }
    const uint4 *const from = reinterpret_cast<const uint4 *>(is_v ? a.v_new : a.k_new);
    const int64_t row_bytes = (int64_t)hk * D;
    // LDS works a wave's accesses off in order: this only keeps the compiler from changing that order
    auto in_order = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); };

    for (; runs; runs &= runs - 1) {
        const int at = __builtin_ctzll(runs);
        const uint64_t after = at == 63 ? 0 : begins >> (at + 1);
        const int end = after ? at + 1 + __builtin_ctzll(after) : 64;
        const int blk = __builtin_amdgcn_readlane(my_blk, at);
        const int64_t block0 = (int64_t)blk << a.block_log2;
        const int base = (int)block0;                       // positions are 32 bits
        float *const scale_at = (is_v ? a.v_scale : a.k_scale) + (int64_t)blk * hk + g;
        const float old = inside ? *scale_at : 0.f;

        in_order();
        src[lane] = -1;
        src[lane + 64] = -1;
        in_order();
        if (lane >= at && lane < end && my_blk >= 0) atomicMax(&src[my_pos - base], (int)(chunk0 + lane));
        // the run's entries among the n times 64 from s on; whether it may go on behind them
        auto follow = [&](int64_t s, auto n) -> bool {
            const int32_t *const at = a.sel_pos + s;
            const int there = (int)min(a.n_sel - s, (int64_t)(n * kWave));
            int p[n];
            bool on = true;
#pragma unroll
            for (int j = 0; j < n; ++j) p[j] = j * kWave + lane < there ? at[j * kWave + lane] : -1;
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const int b = blk_of(p[j]);
                const uint64_t out = __ballot(b >= 0 && b != blk);
                if (on && lane < (out ? __builtin_ctzll(out) : 64) && b >= 0) atomicMax(&src[p[j] - base], (int)(s + j * kWave + lane));
                on = on && !out;
            }
            return on && s + n * kWave < a.n_sel;
        };
        if (end == 64 && chunk0 + 64 < a.n_sel && follow(chunk0 + 64, std::integral_constant<int, 1>{}))
            for (int64_t s = chunk0 + 128; follow(s, std::integral_constant<int, kSkips>{});) s += kSkips * kWave;
        in_order();
        const int rows_here = (int)min((int64_t)1 << a.block_log2, a.n_rows - block0);
        const uint64_t lo = __ballot(src[lane] >= 0), hi = __ballot(src[lane + 64] >= 0);
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        if ((lo >> lane) & 1) row_at[__popcll(lo & below)] = lane;
        if ((hi >> lane) & 1) row_at[__popcll(lo) + __popcll(hi & below)] = lane + 64;
        in_order();
        const int count = __popcll(lo) + __popcll(hi);
        const bool keeps = count < rows_here;
        uint8_t *const to = (is_v ? a.v : a.k) + block0 * row_bytes;

        uint4 w[kListRows];
        uint32_t bits = 0;
        auto load = [&](int k0) {                           // rows k0 .. k0 + 7 of the run; beyond its end: zeros
#pragma unroll
            for (int j = 0; j < kListRows; ++j) {
                w[j] = make_uint4(0u, 0u, 0u, 0u);
                if (k0 + j < count && inside) w[j] = from[(int64_t)src[row_at[k0 + j]] * pieces + piece];
            }
        };
        for (int k0 = 0; k0 < count; k0 += kListRows) {
            load(k0);
#pragma unroll
            for (int j = 0; j < kListRows; ++j) bits = max(bits, magnitude_bits<DTYPE>(w[j]));
        }
        bits = head_max_bits<PPR>(bits);
        const NewScale n = new_scale<CODE>(bits, old, keeps);
        for (int k0 = 0; k0 < count; k0 += kListRows) {
            if (count > kListRows) load(k0);                // (a long run: a second time)
#pragma unroll
            for (int j = 0; j < kListRows; ++j)
                if (k0 + j < count && inside) write_codes<DTYPE, CODE>(to + row_at[k0 + j] * row_bytes + piece * E, w[j], n.inv, n.odd);
        }
        if (inside && lane % PPR == 0) *scale_at = n.scale;
        // Kept rows stand for what they stood for, in steps of the new scale: head by head, 64 pieces of 16 codes of it at once.
        constexpr int kCodes = D / 16, kAtOnce = kWave / kCodes;
        for (uint64_t need = __ballot(n.again && inside && lane % PPR == 0); need; need &= need - 1) {
            const int of = __builtin_ctzll(need);
            const float ratio = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(n.ratio), of));
            uint8_t *const codes = to + (piece - lane + of) * E + (lane % kCodes) * 16;
            for (int r0 = lane / kCodes; r0 < rows_here; r0 += kAgain * kAtOnce) {
                uint4 x[kAgain];
#pragma unroll
                for (int j = 0; j < kAgain; ++j) {
                    const int r = r0 + j * kAtOnce;
                    x[j] = make_uint4(0u, 0u, 0u, 0u);
                    if (r < rows_here && src[r] < 0) x[j] = *reinterpret_cast<const uint4 *>(codes + r * row_bytes);
                }
#pragma unroll
                for (int j = 0; j < kAgain; ++j) {
                    const int r = r0 + j * kAtOnce;
                    if (r < rows_here && src[r] < 0)
                        *reinterpret_cast<uint4 *>(codes + r * row_bytes) =
                            make_uint4(again4<CODE>(x[j].x, ratio), again4<CODE>(x[j].y, ratio), again4<CODE>(x[j].z, ratio), again4<CODE>(x[j].w, ratio));
                }
            }
        }
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
    dim3 grid;
    if (sel_pos) {
        // how many runs the list has is not known here: as many as if its rows were drawn from the cache
        const double blocks = (double)((cache->n_rows + block - 1) / block), runs = blocks * (1.0 - exp(-(double)n_sel / blocks));
        const int64_t pieces = (int64_t)shape->n_kv_heads * shape->head_dim * (int64_t)elem_bytes(shape->dtype) / 16, groups = 2 * ((pieces + kWave - 1) / kWave);
        int64_t chunk = 1;
        while (chunk < kMaxChunk && (3 * chunk * runs <= (double)n_sel || (n_sel / chunk) * groups > kManyWaves)) chunk *= 2;
        a.chunk = (int)chunk;
        grid = dim3((unsigned)((n_sel + 4 * chunk - 1) / (4 * chunk)), (unsigned)groups);
    } else {
        // 1024 workgroups keep the compute units busy, and a block has no more rounds to share
        const int64_t wgs = (row0 + n_sel - 1) / block - row0 / block + 1;
        const int64_t rounds = (units + teams - 1) / teams;
        int64_t split = (1024 + wgs - 1) / wgs;
        if (split > rounds) split = rounds;
        a.units_per_wg = (int)((rounds + split - 1) / split) * teams;
        grid = dim3((unsigned)wgs, (unsigned)((units + a.units_per_wg - 1) / a.units_per_wg));
    }
    if (grid.x > (unsigned)kMostWgs) return fail(KVS_EUNSUPPORTED, "kvs_store_kv8: %lld rows in one call", (long long)n_sel);
    hipStream_t hs = (hipStream_t)stream;
#define KVS_STORE(DT, C, DD)                                                                                          \
    do {                                                                                                              \
        if (sel_pos) hipLaunchKernelGGL((store_list_kernel<DT, C, DD>), grid, dim3(kThreads), 0, hs, a);               \
        else hipLaunchKernelGGL((store_rows_kernel<DT, C, DD>), grid, dim3(kThreads), 0, hs, a);                       \
    } while (0)
#define KVS_STORE_D(DT, C) do { if (shape->head_dim == 128) KVS_STORE(DT, C, 128); else KVS_STORE(DT, C, 64); } while (0)
    if (shape->dtype == KVS_BF16) { if (cache->code == KVS_E4M3) KVS_STORE_D(KVS_BF16, KVS_E4M3); else KVS_STORE_D(KVS_BF16, KVS_INT8); }
    else { if (cache->code == KVS_E4M3) KVS_STORE_D(KVS_F32, KVS_E4M3); else KVS_STORE_D(KVS_F32, KVS_INT8); }
#undef KVS_STORE_D
#undef KVS_STORE
    return check_launch("kvs_store_kv8");
}
