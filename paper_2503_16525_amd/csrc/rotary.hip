// kvs_rotary: the rotary positions of Q and K rows, fresh ones or reused ones that move to another position.
//
// A pair (u, v) of channels turns by a = (pos - pos_from) * f_j.  The frequencies are made on the host in fp64 (up to 64
// of them, passed by value, in turns per position), the angle is formed in fp64 on the device, reduced to its fraction of a
// turn there, and only that fraction goes to fp32: at position 10^6 the angle is good to 1e-7 and sine and cosine to that.
//
// What bounds it is memory: every element is read and written once, with three flops.  Sine and cosine of a (token,
// pair) are the same for all heads, so a workgroup takes a few tokens, makes their sines and cosines once, one pair a
// thread, into LDS (8 bytes a pair), and then streams the tokens' heads: a thread takes a cell of 16 bytes of u and 16 bytes
// of v (in the interleaved layout, and where channels pass through to another buffer, 32 bytes in a row).  What a cell is is found
// by multiplications, and a thread has one cell at a time: with divisions and two cells, 131072 rows of 4 heads took 74 us instead
// of 52 to 54, which is what a copy of their bytes takes; 8192 rows of 32 + 8 heads 39 instead of 30 (5.5 TB/s; 34 with ordinary loads).
// Both layouts need rotary_dim to be a multiple of two cells' channels (16 in bf16, 8 in fp32); other sizes go to a
// kernel that takes one pair a thread and makes its angle for every head anew: 8192 rows of 32 + 8 heads with 100 channels turned 92 us, with 2 to 36
// of them 117 to 125, where cells take 29 to 35.  Turned parts of such sizes are rare, and the kernel is kept short.
#include "kvs_internal.h"

#include <math.h>

#include <type_traits>

namespace kvs {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 64;
constexpr int kMostHeads = 4095;      // of Q and K together
constexpr int kMaxTokens = 32;        // tokens a workgroup takes at most: 16 KiB of sines and cosines

struct Frequencies { double turns[kMaxPairs]; };   // per position

// One of q, k: where its rows lie.
struct Rows {
    const void *in;
    void *out;
    int64_t in_stride, out_stride;      // elements
    int32_t heads;
};

// x / n for x * n below 2^32
struct Divisor {
    uint32_t n, m;
    explicit Divisor(uint32_t d) : n(d), m(d > 1 ? (uint32_t)((((uint64_t)1 << 32) + d - 1) / d) : 0u) {}
    __device__ __forceinline__ int operator()(int x) const { return n > 1 ? (int)__umulhi((uint32_t)x, m) : x; }
};

__device__ __forceinline__ float2 turn_of(double turns)
{
    const float part = (float)(turns - rint(turns));     // -0.5 .. 0.5 of a turn
    float s, c;
    sincospif(2.f * part, &s, &c);
    return make_float2(c, s);
}

__device__ __forceinline__ double moved(const int32_t *pos, const int32_t *pos_from, int64_t i)
{
    return (double)pos[i] - (pos_from ? (double)pos_from[i] : 0.0);
}

template <int DTYPE> struct Cell;                        // 16 bytes
template <> struct Cell<KVS_BF16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void widen(const uint4 w, float (&x)[E])
    {
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    }
    static __device__ __forceinline__ uint4 round(const float (&x)[E])
    {
        return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
};
template <> struct Cell<KVS_F32> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void widen(const uint4 w, float (&x)[E])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint4 round(const float (&x)[E])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// cells of one head: pairs of 16-byte pieces, those that turn, then, where the output is another buffer, those that pass through
template <int DTYPE, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const Frequencies fr, const Rows q, const Rows k, int64_t n_tokens, int tokens_per_wg,
                                                          const Divisor pairs_d, const Divisor per_token_d, const Divisor per_head_d, int cells_q, int head_dim, float magnitude,
                                                          const int32_t *__restrict__ pos, const int32_t *__restrict__ pos_from)
{
    constexpr int E = Cell<DTYPE>::E;
    extern __shared__ float2 cs[];                         // [tokens][pairs] (cos, sin), times the magnitude
    const int tid = threadIdx.x, pairs = (int)pairs_d.n;
    const int64_t tok0 = (int64_t)blockIdx.x * tokens_per_wg;
    const int toks = (int)min((int64_t)tokens_per_wg, n_tokens - tok0);
    for (int e = tid; e < toks * pairs; e += kThreads) {
        const int t = pairs_d(e), j = e - t * pairs;
        const float2 x = turn_of(moved(pos, pos_from, tok0 + t) * fr.turns[j]);
        cs[e] = make_float2(x.x * magnitude, x.y * magnitude);
    }
    __syncthreads();

    const int turned = pairs / E, per_head = (int)per_head_d.n, per_token = (int)per_token_d.n, all = toks * per_token;
    for (int c = tid; c < all; c += kThreads) {
        const int t = per_token_d(c);
        int cell = c - t * per_token;
        const bool is_k = cell >= cells_q;
        if (is_k) cell -= cells_q;
        const int head = per_head_d(cell), piece = cell - head * per_head;
        const bool turns = piece < turned;
        // first channels of the cell's two pieces (2 E turned channels to a cell that turns, so the others begin at 2 E turned)
        const int c0 = INTERLEAVED || !turns ? 2 * E * piece : E * piece, c1 = INTERLEAVED || !turns ? c0 + E : c0 + pairs;
        const int64_t row = tok0 + t;
        constexpr int size = 16 / E;
        const char *in = (const char *)(is_k ? k.in : q.in) + (row * (is_k ? k.in_stride : q.in_stride) + (int64_t)head * head_dim) * size;
        char *out = (char *)(is_k ? k.out : q.out) + (row * (is_k ? k.out_stride : q.out_stride) + (int64_t)head * head_dim) * size;
        const uint4 a = stream_load16(reinterpret_cast<const uint4 *>(in + c0 * size)), b = stream_load16(reinterpret_cast<const uint4 *>(in + c1 * size));
        uint4 *const to_a = reinterpret_cast<uint4 *>(out + c0 * size), *const to_b = reinterpret_cast<uint4 *>(out + c1 * size);
        if (!turns) { *to_a = a; *to_b = b; continue; }
        const float2 *const at = cs + t * pairs + piece * E;
        float x[E], y[E], xx[E], yy[E];
        Cell<DTYPE>::widen(a, x);
        Cell<DTYPE>::widen(b, y);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float2 r = at[e];
            // interleaved: pair e is channels 2e, 2e + 1 of the 2E in a row
            const float u = INTERLEAVED ? (e < E / 2 ? x[2 * e % E] : y[2 * e % E]) : x[e];
            const float v = INTERLEAVED ? (e < E / 2 ? x[(2 * e + 1) % E] : y[(2 * e + 1) % E]) : y[e];
            const float uu = u * r.x - v * r.y, vv = v * r.x + u * r.y;
            if (!INTERLEAVED) { xx[e] = uu; yy[e] = vv; }
            else if (e < E / 2) { xx[2 * e % E] = uu; xx[(2 * e + 1) % E] = vv; }
            else { yy[2 * e % E] = uu; yy[(2 * e + 1) % E] = vv; }
        }
        *to_a = Cell<DTYPE>::round(xx);
        *to_b = Cell<DTYPE>::round(yy);
    }
}

// any even rotary_dim: a thread takes one pair, or one channel that passes through
template <int DTYPE>
__global__ __launch_bounds__(kThreads) void rotary_pairs_kernel(const Frequencies fr, const Rows x, int64_t n_items, int pairs, int per_head, int head_dim,
                                                                int interleaved, float magnitude, const int32_t *__restrict__ pos,
                                                                const int32_t *__restrict__ pos_from)
{
    const int64_t it = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (it >= n_items) return;
    const int j = (int)(it % per_head);
    const int64_t cell = it / per_head, row = cell / x.heads;
    const int head = (int)(cell % x.heads);
    const int64_t in = row * x.in_stride + (int64_t)head * head_dim, out = row * x.out_stride + (int64_t)head * head_dim;
    using T = typename std::conditional<DTYPE == KVS_BF16, uint16_t, float>::type;
    const T *src = (const T *)x.in + in;
    T *dst = (T *)x.out + out;
    if (j >= pairs) {                                     // only where the output is another buffer
        dst[j + pairs] = src[j + pairs];
        return;
    }
    const float2 r = turn_of(moved(pos, pos_from, row) * fr.turns[j]);
    const int c0 = interleaved ? 2 * j : j, c1 = interleaved ? c0 + 1 : c0 + pairs;
    auto widen = [](T v) -> float { if constexpr (DTYPE == KVS_BF16) return bf16_lo(v); else return v; };
    const float u = widen(src[c0]), v = widen(src[c1]);
    const float c = r.x * magnitude, s = r.y * magnitude;
    const float uu = u * c - v * s, vv = v * c + u * s;
    if constexpr (DTYPE == KVS_BF16) { dst[c0] = (uint16_t)f32_to_bf16_bits(uu); dst[c1] = (uint16_t)f32_to_bf16_bits(vv); }
    else { dst[c0] = uu; dst[c1] = vv; }
}

kvs_status check_spec(const kvs_rotary_spec *sp, int head_dim)
{
    const char *me = "kvs_rotary";
    if (!sp) return fail(KVS_EINVAL, "%s: spec is NULL", me);
    if (sp->rotary_dim < 2 || sp->rotary_dim > head_dim || (sp->rotary_dim & 1))
        return fail(KVS_EINVAL, "%s: rotary_dim %d is not even and within 2 .. head_dim %d", me, sp->rotary_dim, head_dim);
    if (sp->layout != KVS_ROTARY_HALF && sp->layout != KVS_ROTARY_INTERLEAVED) return fail(KVS_EINVAL, "%s: unknown layout %d", me, sp->layout);
    if (sp->scaling < KVS_ROTARY_PLAIN || sp->scaling > KVS_ROTARY_WAVELENGTH) return fail(KVS_EINVAL, "%s: unknown scaling %d", me, sp->scaling);
    if (!(sp->base > 1.0) || !isfinite(sp->base)) return fail(KVS_EINVAL, "%s: base %g is not above 1", me, sp->base);
    if (!isfinite((float)sp->magnitude)) return fail(KVS_EINVAL, "%s: the magnitude is not finite", me);
    if (sp->scaling == KVS_ROTARY_PLAIN) return KVS_OK;
    if (!(sp->factor > 0.0) || !isfinite(sp->factor)) return fail(KVS_EINVAL, "%s: factor %g is not above 0", me, sp->factor);
    if (sp->scaling == KVS_ROTARY_NTK && sp->rotary_dim == 2) return fail(KVS_EINVAL, "%s: the base cannot be stretched for a single pair", me);
    if (sp->scaling == KVS_ROTARY_RAMP || sp->scaling == KVS_ROTARY_WAVELENGTH) {
        if (sp->original <= 0) return fail(KVS_EINVAL, "%s: original context length %d", me, sp->original);
        if (!(sp->low > 0.0) || !(sp->high > sp->low) || !isfinite(sp->high)) return fail(KVS_EINVAL, "%s: turns %g .. %g are not 0 < low < high", me, sp->low, sp->high);
    }
    return KVS_OK;
}

Frequencies frequencies(const kvs_rotary_spec &sp)
{
    const double two_pi = 6.283185307179586476925286766559;
    Frequencies fr = {};
    const int r = sp.rotary_dim, pairs = r / 2;
    double log_base = log(sp.base);
    if (sp.scaling == KVS_ROTARY_NTK) log_base += log(sp.factor) * r / (r - 2.0);
    double first = 0.0, last = 0.0;
    if (sp.scaling == KVS_ROTARY_RAMP) {
        first = fmax(floor(r * log(sp.original / (sp.high * two_pi)) / (2.0 * log_base)), 0.0);
        last = fmin(ceil(r * log(sp.original / (sp.low * two_pi)) / (2.0 * log_base)), r - 1.0);
    }
    for (int j = 0; j < pairs; ++j) {
        double f = exp(-2.0 * j / r * log_base) / two_pi;
        if (sp.scaling == KVS_ROTARY_LINEAR) f /= sp.factor;
        if (sp.scaling == KVS_ROTARY_RAMP) {
            const double w = fmin(fmax((j - first) / fmax(last - first, 0.001), 0.0), 1.0);
            f = f * (1.0 - w) + f / sp.factor * w;
        }
        if (sp.scaling == KVS_ROTARY_WAVELENGTH) {
            const double w = fmin(fmax((sp.original * f - sp.low) / (sp.high - sp.low), 0.0), 1.0);
            f = f * w + f / sp.factor * (1.0 - w);
        }
        fr.turns[j] = f;
    }
    return fr;
}

// n rows of `row` bytes, `stride` bytes apart
struct Slab { uintptr_t at; int64_t stride, row; };
Slab slab_of(const void *p, int64_t stride, const Rows &x, int head_dim, size_t size)
{
    return {reinterpret_cast<uintptr_t>(p), stride * (int64_t)size, (int64_t)x.heads * head_dim * (int64_t)size};
}

// Whether two of them have a byte in common.  With one stride that is exact: rows may lie beside each other in one buffer.  With two, what
// lies between the other's first and last row is taken to.
bool overlap(const Slab &a, const Slab &b, int64_t n)
{
    const uintptr_t a_end = a.at + (uintptr_t)((n - 1) * a.stride + a.row), b_end = b.at + (uintptr_t)((n - 1) * b.stride + b.row);
    if (a_end <= b.at || b_end <= a.at) return false;
    if (n == 1 || a.stride != b.stride) return true;
    // row j of b begins d bytes behind row j + k of a, which exists for some j if -n < k < n
    const int64_t apart = (int64_t)(b.at - a.at), k = apart >= 0 ? apart / a.stride : -((-apart + a.stride - 1) / a.stride), d = apart - k * a.stride;
    auto exists = [n](int64_t rows) { return rows > -n && rows < n; };
    return (d < a.row && exists(k)) || (d + b.row > a.stride && exists(k + 1));
}

kvs_status check_rows(const char *name, const Rows &x, int64_t n, int head_dim, size_t size)
{
    const int64_t row = (int64_t)x.heads * head_dim, step = 16 / (int64_t)size;
    if (!x.in || !x.out) return fail(KVS_EINVAL, "kvs_rotary: %s or %s_out is NULL", name, name);
    if (!aligned16(x.in) || !aligned16(x.out)) return fail(KVS_EINVAL, "kvs_rotary: %s and %s_out must be 16-byte aligned", name, name);
    if (x.in_stride < row || x.out_stride < row || x.in_stride % step || x.out_stride % step)
        return fail(KVS_EINVAL, "kvs_rotary: strides %lld, %lld of %s: at least a row of %lld elements and a multiple of %lld", (long long)x.in_stride,
                    (long long)x.out_stride, name, (long long)row, (long long)step);
    const int64_t most = x.in_stride > x.out_stride ? x.in_stride : x.out_stride;
    if (n > ((int64_t)1 << 46) / most) return fail(KVS_EINVAL, "kvs_rotary: %lld rows %lld elements apart", (long long)n, (long long)most);
    return KVS_OK;
}

} // namespace
} // namespace kvs

extern "C" kvs_status kvs_rotary(const kvs_shape *shape, const kvs_rotary_spec *spec, int64_t n_tokens,
                                 const int32_t *pos, const int32_t *pos_from,
                                 const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                 void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream)
{
    using namespace kvs;
    kvs_status st = check_shape(shape);
    if (st != KVS_OK) return st;
    const int d = shape->head_dim;
    // a token's cells, at most 16 a head, stay below 2^16 (Divisor)
    if ((int64_t)shape->n_q_heads + shape->n_kv_heads > kMostHeads) return fail(KVS_EUNSUPPORTED, "kvs_rotary: more than %d heads", kMostHeads);
    if ((st = check_spec(spec, d)) != KVS_OK) return st;
    if (n_tokens < 0) return fail(KVS_EINVAL, "kvs_rotary: n_tokens < 0");
    if (n_tokens == 0) return KVS_OK;
    if (!pos) return fail(KVS_EINVAL, "kvs_rotary: pos is NULL");
    const size_t size = elem_bytes(shape->dtype);
    Rows rows[2] = {{q, q_out, q_stride, q_out_stride, shape->n_q_heads}, {k, k_out, k_stride, k_out_stride, shape->n_kv_heads}};
    if (!q && !k) return fail(KVS_EINVAL, "kvs_rotary: neither q nor k is given");
    for (int i = 0; i < 2; ++i) {
        if (!rows[i].in) { rows[i].heads = 0; continue; }
        if ((st = check_rows(i ? "k" : "q", rows[i], n_tokens, d, size)) != KVS_OK) return st;
    }
    const char *const names[2] = {"q", "k"};
    for (int i = 0; i < 2; ++i) {
        if (!rows[i].heads) continue;
        const Slab out = slab_of(rows[i].out, rows[i].out_stride, rows[i], d, size);
        for (int j = 0; j < 2; ++j) {
            if (!rows[j].heads) continue;
            const Slab in = slab_of(rows[j].in, rows[j].in_stride, rows[j], d, size), other = slab_of(rows[j].out, rows[j].out_stride, rows[j], d, size);
            const bool in_place = i == j && in.at == out.at && (n_tokens == 1 || in.stride == out.stride);
            if (!in_place && overlap(out, in, n_tokens)) return fail(KVS_EINVAL, "kvs_rotary: %s_out overlaps %s without being in place", names[i], names[j]);
            if (i < j && overlap(out, other, n_tokens)) return fail(KVS_EINVAL, "kvs_rotary: %s_out overlaps %s_out", names[i], names[j]);
        }
    }
    const Frequencies fr = frequencies(*spec);
    const int pairs = spec->rotary_dim / 2, e = 16 / (int)size, left = d - spec->rotary_dim;
    const float magnitude = (float)spec->magnitude;
    hipStream_t hs = (hipStream_t)stream;
    const bool bf16 = shape->dtype == KVS_BF16;
    // rows turned in place leave what passes through where it is
    auto in_place = [](const Rows &x) { return x.in == x.out; };
    const bool same = (!rows[0].heads || in_place(rows[0])) && (!rows[1].heads || in_place(rows[1]));
    if (pairs % e == 0) {
        const int per_head = pairs / e + (same ? 0 : left / (2 * e));
        const int cells_q = rows[0].heads * per_head, cells_k = rows[1].heads * per_head, per_token = cells_q + cells_k;
        // as many tokens as give every thread a cell, as long as that leaves two workgroups a compute unit
        int toks = (kThreads + per_token - 1) / per_token;
        if (toks > kMaxTokens) toks = kMaxTokens;
        if (toks > n_tokens / 512) toks = (int)(n_tokens / 512);
        if (toks < 1) toks = 1;
        const int64_t wgs = (n_tokens + toks - 1) / toks;
        if (wgs > kMostWgs) return fail(KVS_EUNSUPPORTED, "kvs_rotary: %lld rows in one call", (long long)n_tokens);
        const size_t lds = (size_t)toks * pairs * sizeof(float2);
#define KVS_ROT(DT, IL)                                                                                                              \
        hipLaunchKernelGGL((rotary_kernel<DT, IL>), dim3((unsigned)wgs), dim3(kThreads), lds, hs, fr, rows[0], rows[1], n_tokens, toks,       \
                           Divisor(pairs), Divisor(per_token), Divisor(per_head), cells_q, d, magnitude, pos, pos_from)
        const bool il = spec->layout == KVS_ROTARY_INTERLEAVED;
        if (bf16) { if (il) KVS_ROT(KVS_BF16, true); else KVS_ROT(KVS_BF16, false); }
        else { if (il) KVS_ROT(KVS_F32, true); else KVS_ROT(KVS_F32, false); }
#undef KVS_ROT
        return check_launch("kvs_rotary");
    }
    for (int i = 0; i < 2; ++i) {
        if (!rows[i].heads) continue;
        const int per_head = pairs + (in_place(rows[i]) ? 0 : left);
        const int il = spec->layout == KVS_ROTARY_INTERLEAVED;
        const int64_t most = kMostWgs * kThreads / (rows[i].heads * per_head);          // rows of a launch
        for (int64_t t0 = 0; t0 < n_tokens; t0 += most) {
            const int64_t n = n_tokens - t0 < most ? n_tokens - t0 : most, items = n * rows[i].heads * per_head, wgs = (items + kThreads - 1) / kThreads;
            Rows x = rows[i];
            x.in = (const char *)x.in + t0 * x.in_stride * (int64_t)size;
            x.out = (char *)x.out + t0 * x.out_stride * (int64_t)size;
            const int32_t *from = pos_from ? pos_from + t0 : nullptr;
            if (bf16) hipLaunchKernelGGL((rotary_pairs_kernel<KVS_BF16>), dim3((unsigned)wgs), dim3(kThreads), 0, hs, fr, x, items, pairs, per_head, d, il, magnitude, pos + t0, from);
            else hipLaunchKernelGGL((rotary_pairs_kernel<KVS_F32>), dim3((unsigned)wgs), dim3(kThreads), 0, hs, fr, x, items, pairs, per_head, d, il, magnitude, pos + t0, from);
            if ((st = check_launch("kvs_rotary")) != KVS_OK) return st;
        }
    }
    return KVS_OK;
}
