// What the kernels over an 8-bit cache share: how codes are read and written (not part of the ABI).
#pragma once

#include "kvs_internal.h"

namespace kvs {

// Checks a cache description against the shape; `me` names the call.
kvs_status check_cache8(const char *me, const kvs_shape *shape, const kvs_cache8 *cache);
size_t attention8_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t n_rows_total, int64_t n_sel_total);

constexpr float kLeastScale = 1.1754943508222875e-38f;    // 2^-126: 1 / scale stays finite

template <int CODE> __host__ __device__ constexpr float top_code() { return CODE == KVS_E4M3 ? 448.f : 127.f; }

// e4m3's two NaN codes (0x7f, 0xff) of four codes become the largest numbers: memory that no store wrote can hold them, and a
// weight of 0 does not hide a NaN.
__device__ __forceinline__ uint32_t numbers_only(uint32_t w)
{
    const uint32_t t = (w & 0x7f7f7f7fu) + 0x01010101u;       // 0x80 in the bytes that are NaN
    return w - ((t >> 7) & 0x01010101u);
}

// four codes as fp32, exactly
template <int CODE>
__device__ __forceinline__ void widen_codes(uint32_t w, float (&x)[4])
{
    if constexpr (CODE == KVS_E4M3) {
        x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
        x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
        x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
        x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
    } else {
        x[0] = (float)(int8_t)(w & 0xffu);
        x[1] = (float)(int8_t)((w >> 8) & 0xffu);
        x[2] = (float)(int8_t)((w >> 16) & 0xffu);
        x[3] = (float)(int8_t)(w >> 24);
    }
}

// The nearest codes (ties to even) to four numbers times `by`, products that pass the largest code by their rounding at most.
template <int CODE>
__device__ __forceinline__ uint32_t nearest_codes(float a, float b, float c, float d, float by)
{
#pragma clang fp contract(off)
    if constexpr (CODE == KVS_E4M3) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * by, b * by, 0, false);          // (up to 464 the nearest is 448)
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * by, d * by, w, true);
    } else {
        // 1.5 * 2^23 + x, rounded, ends with the whole number nearest to x in two's complement
        const float m = 12582912.f;
        const uint32_t x = __float_as_uint(a * by + m), y = __float_as_uint(b * by + m), z = __float_as_uint(c * by + m), w = __float_as_uint(d * by + m);
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w, z, 0x0c0c0400u), __builtin_amdgcn_perm(y, x, 0x0c0c0400u), 0x05040100u);
    }
}

} // namespace kvs
