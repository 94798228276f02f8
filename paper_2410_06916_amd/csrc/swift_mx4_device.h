// Device code that the MXFP4 kernels share: codes to numbers, and what follows a call's dot products.
#pragma once
#include <math.h>

#include "swift_device.h"
#include "swift_mx4.h"

namespace swift {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight codes to the eight bf16 values they stand for (exact): an A operand.
__device__ inline bf16x8 mx4_decode(uint32_t w, float scale) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
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
// Values [row, row + n) of row r, 0 <= n <= 4; vec: as mx4_out_by_fours says.
__device__ inline f32x4 mx4_residual4(const Mx4Out &o, int r, int row, int n, bool vec) {
    const int64_t at = r * o.ld_res + row;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (vec && n == 4) {
        if (o.dtype == F32) {
            v = *(const f32x4 *)((const float *)o.residual + at);
        } else {
            const uint64_t w = *(const uint64_t *)((const uint16_t *)o.residual + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float((uint32_t)(w >> (16 * i)) << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) v[i] = load_as_f32(o.residual, o.dtype, at + i);
    }
    return v;
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

// What follows the dot products of one row group of a call, by thread t of `threads`.  Y(r, j): row r's product with tile row j.
template <int EPI, typename YF>
__device__ inline void mx4_call_epilogue(const Mx4Out &o, int R, int O, int rg, int t, int threads, YF Y) {
    if (EPI == EPI_LINEAR) {
        for (int i = t; i < 16 * R; i += threads) {
            const int r = i >> 4, row = 16 * rg + (i & 15);
            if (row >= O) continue;
            float y = Y(r, i & 15);
            if (o.residual) y += load_as_f32(o.residual, o.dtype, r * o.ld_res + row);
            store_f32_as(o.y, o.dtype, r * o.ld + row, y);
        }
    } else {
        for (int i = t; i < 8 * R; i += threads) {
            const int r = i >> 3, j = i & 7, row = 8 * rg + j;
            if (row >= O) continue;
            const float g = Y(r, j), u = Y(r, j + 8);
            store_f32_as(o.y, o.dtype, r * o.ld + row, mx4_silu(g) * u);
        }
    }
}

}  // namespace swift
