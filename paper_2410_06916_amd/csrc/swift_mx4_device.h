// Device code that the MXFP4 kernels share: codes to numbers, and what follows a call's dot products.
#pragma once
#include <math.h>

#include <type_traits>
#include <utility>

#include "swift_device.h"
#include "swift_mx4.h"

namespace swift {

// f(0), f(1), .. f(N - 1), each a constant.
template <int N, typename F, int... I>
__device__ inline void each_of(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ inline void each(F &&f) {
    each_of<N>(f, std::make_integer_sequence<int, N>());
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight codes to the eight bf16 values they stand for (exact): an A operand.
__device__ inline bf16x8 mx4_decode(uint32_t w, float scale) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// Elements k0 .. k0 + 7 of a row as fp32, zeros past K.  vec: the row allows 16-byte loads.
template <typename T>
__device__ inline void mx4_load8(const typename T::elem *row, int k0, int K, bool vec, float *v) {
    if (vec && k0 + 8 <= K) {
#pragma unroll
        for (int i = 0; i < 8; i += T::VEC) T::unpack(*(const u32x4 *)(row + k0 + i), v + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k0 + i < K ? T::load1(row + k0 + i) : 0.f;
    }
}

// v = hi + mid + lo exactly, for every finite v: hi is cut off, so that it never overflows.  Infinities and NaNs have one term.
__device__ inline void mx4_split3(float v, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
    const uint32_t u = __float_as_uint(v);
    hi = u >> 16;
    mid = lo = 0;
    if ((u & 0x7f800000u) == 0x7f800000u) {
        if (u & 0x007fffffu) hi |= 0x40u;
        return;
    }
    const float r = v - __uint_as_float(hi << 16);
    mid = f32_to_bf16_rne_finite(r);
    lo = f32_to_bf16_rne_finite(r - __uint_as_float(mid << 16));
}

// Eight values to three units of eight bf16, a term each.
__device__ inline void mx4_split8(const float *v, u32x4 (&t)[3]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h[2], m[2], l[2];
        mx4_split3(v[2 * i], h[0], m[0], l[0]);
        mx4_split3(v[2 * i + 1], h[1], m[1], l[1]);
        t[0][i] = pack2(h[0], h[1]);
        t[1][i] = pack2(m[0], m[1]);
        t[2][i] = pack2(l[0], l[1]);
    }
}

__device__ inline float load_as_f32(const void *p, int dtype, int64_t i) {
    return dtype == F32 ? ((const float *)p)[i] : BF16T::load1((const uint16_t *)p + i);
}
__device__ inline void store_f32_as(void *p, int dtype, int64_t i, float v) {
    if (dtype == F32)
        ((float *)p)[i] = v;
    else
        ((uint16_t *)p)[i] = f32_to_bf16_rne(v);  // (the result's one rounding)
}

__device__ inline float mx4_silu(float g) { return g / (1.0f + expf(-g)); }

// The result from row r0 on.
__device__ inline Mx4Out mx4_out_from(Mx4Out o, int64_t r0) {
    const int64_t eb = o.dtype == F32 ? 4 : 2;
    o.y = (char *)o.y + r0 * o.ld * eb;
    if (o.residual) o.residual = (const char *)o.residual + r0 * o.ld_res * eb;
    return o;
}
// Whether four values that start at a multiple of four of a row can be moved at once.
__device__ inline bool mx4_out_by_fours(const Mx4Out &o) {
    const uintptr_t bits = o.dtype == F32 ? 15 : 7;
    return ((uintptr_t)o.y & bits) == 0 && (o.ld & 3) == 0 && (!o.residual || (((uintptr_t)o.residual & bits) == 0 && (o.ld_res & 3) == 0));
}
// Residual values [row, row + n) of row r, 0 <= n <= 4, as they are loaded (vec, as mx4_out_by_fours says, and all four: the words in memory, so that nothing
// waits for them here; else fp32), and as numbers.
__device__ inline u32x4 mx4_residual_words(const Mx4Out &o, int r, int row, int n, bool vec) {
    const int64_t at = r * o.ld_res + row;
    u32x4 w = {0u, 0u, 0u, 0u};
    if (vec && n == 4) {
        if (o.dtype == F32) {
            w = *(const u32x4 *)((const float *)o.residual + at);
        } else {
            const uint2 b = *(const uint2 *)((const uint16_t *)o.residual + at);
            w[0] = b.x;
            w[1] = b.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) w[i] = __float_as_uint(load_as_f32(o.residual, o.dtype, at + i));
    }
    return w;
}
__device__ inline f32x4 mx4_residual_values(const Mx4Out &o, const u32x4 &w, int n, bool vec) {
    if (o.dtype == F32 || !(vec && n == 4)) return __builtin_bit_cast(f32x4, w);
    return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
}
__device__ inline void mx4_store4(const Mx4Out &o, int r, int row, int n, bool vec, const f32x4 &v) {
    const int64_t at = r * o.ld + row;
    if (vec && n == 4) {
        if (o.dtype == F32) {
            *(f32x4 *)((float *)o.y + at) = v;
        } else {  // (the results' one rounding)
            uint64_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w |= (uint64_t)f32_to_bf16_rne(v[i]) << (16 * i);
            *(uint64_t *)((uint16_t *)o.y + at) = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) store_f32_as(o.y, o.dtype, at + i, v[i]);
    }
}

}  // namespace swift
