// MXFP4 matrices: numbers to packed blocks and back, and activations to the B operand's layout (formats: swift_mx4.h).
#include <algorithm>

#include "swift_device.h"
#include "swift_mx4.h"
#include "swift_mx4_device.h"

namespace swift {

namespace {

// Row of the matrix in tile row j of row group rg, or -1: it comes from the other tensor (TILE_GATEUP).
__device__ inline int tile_row(int mode, int part, int d, int rg, int j) {
    if (mode == TILE_PLAIN) return 16 * rg + j;
    if (mode == TILE_GATEUP) return (j >= 8) == (part == 1) ? 8 * rg + (j & 7) : -1;
    const int gph = d >> 4, head = rg / gph, g = rg - head * gph;
    return head * d + 8 * g + (j & 7) + (j >= 8 ? d >> 1 : 0);
}

// One lane per block of 32.  The scale's exponent is that of the largest magnitude less two (its floor(log2) against the four of the largest
// element's binade), at least -127; the conversion instruction divides by the scale, rounds to the nearest element, ties to the even
// code, and saturates at 6, subnormals included.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_quantize(Mx4QuantArgs a, bool vec) {
    const int S = mx4_tiles(a.K);
    const int64_t n = (int64_t)a.n_rg * S * 64;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < n; c += (int64_t)gridDim.x * 256) {
        const int64_t piece = c >> 6;
        const int lane = (int)(c & 63), rg = (int)(piece / S), s = (int)(piece - (int64_t)rg * S);
        const int row = tile_row(a.mode, a.part, a.head_dim, rg, lane & 15), k0 = kMx4Tile * s + kMx4Block * (lane >> 4);
        if (row < 0) continue;
        u32x4 code = {0u, 0u, 0u, 0u};
        uint32_t e = 0;
        if (row < a.src_rows && k0 < a.K) {
            const auto *src = (const typename T::elem *)a.src + (int64_t)row * a.ld;
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; i += 8) mx4_load8<T>(src, k0 + i, a.K, vec, v + i);
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);  // (NaNs above infinity above numbers)
            e = top >> 23;
            if (e != 255) {
                e = e > 2 ? e - 2 : 0;
                const float scale = __uint_as_float(e << 23);  // (the instructions read its exponent field only: 0 is 2^-127)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t q = 0;
                    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w], v[8 * w + 1], scale, 0);
                    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w + 2], v[8 * w + 3], scale, 1);
                    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w + 4], v[8 * w + 5], scale, 2);
                    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w + 6], v[8 * w + 7], scale, 3);
                    code[w] = q;
                }
            }
        }
        ((u32x4 *)a.codes)[c] = code;
        a.scales[c] = (uint8_t)e;
    }
}

template <typename T>
__device__ inline void store8(typename T::elem *row, int k0, int K, bool vec, const float *v) {
    if (vec && k0 + 8 <= K) {
        if constexpr (T::VEC == 8) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
            *(u32x4 *)(row + k0) = w;
        } else {
            *(f32x4 *)(row + k0) = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4 *)(row + k0 + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k0 + i < K) T::store1(row + k0 + i, v[i]);
    }
}

// Eight codes as fp32 (every value is a bf16 number, subnormal ones included: nothing is rounded on the way out).
__device__ inline void decode8(uint32_t w, float scale, float *v) { BF16T::unpack(__builtin_bit_cast(u32x4, mx4_decode(w, scale)), v); }

template <typename T>
__global__ __launch_bounds__(256) void k_mx4_dequantize(Mx4DequantArgs a, bool vec) {
    const int64_t n = (int64_t)a.w.n_rg * a.w.S * 64;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < n; c += (int64_t)gridDim.x * 256) {
        const int64_t piece = c >> 6;
        const int lane = (int)(c & 63), j = lane & 15, rg = (int)(piece / a.w.S), s = (int)(piece - (int64_t)rg * a.w.S);
        const int row = a.mode == TILE_GATEUP ? 8 * rg + (j & 7) : 16 * rg + j, k0 = kMx4Tile * s + kMx4Block * (lane >> 4);
        if (row >= a.rows || k0 >= a.K) continue;
        auto *dst = (typename T::elem *)a.dst + (int64_t)(a.mode == TILE_GATEUP && j >= 8 ? row + a.rows : row) * a.ld;
        const u32x4 code = ((const u32x4 *)a.w.codes)[c];
        const float scale = __uint_as_float((uint32_t)a.w.scales[c] << 23);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            float v[8];
            decode8(code[w], scale, v);
            store8<T>(dst, k0 + 8 * w, a.K, vec, v);
        }
    }
}

// A workgroup turns 64 rows (at most) of a sub-block by 16 chunks through LDS: rows are read 128 k at a time, columns are written a KB at a
// time.  (A thread per chunk that writes where its chunk goes: 512 rows of 4096 bf16 7.5 us.)
constexpr int kActRows = 64;
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_activations(Mx4ActArgs a, int blocks_of_sub, bool vec) {
    constexpr int NT = T::VEC == 8 ? 1 : 3, P = kActRows * NT + 1;
    __shared__ u32x4 turn[16 * P];
    const int s = blockIdx.x, sub = blockIdx.y / blocks_of_sub, b = blockIdx.y - sub * blocks_of_sub;
    const int r0 = sub * a.per + b * kActRows, rows = min(kActRows, min(a.per - b * kActRows, a.n - r0));
    if (rows <= 0) return;
    for (int i = threadIdx.x; i < 16 * rows; i += 256) {
        const int r = i >> 4, ch = i & 15;
        float v[8];
        mx4_load8<T>((const typename T::elem *)a.x + (int64_t)(r0 + r) * a.ld, kMx4Tile * s + 8 * ch, a.K, vec, v);
        u32x4 t[3];
        if constexpr (NT == 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) t[0][j] = (__float_as_uint(v[2 * j]) >> 16) | (__float_as_uint(v[2 * j + 1]) & 0xffff0000u);
        } else {
            mx4_split8(v, t);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) turn[ch * P + NT * r + j] = t[j];
    }
    __syncthreads();
    const int cols = NT * rows;
    u32x4 *out = (u32x4 *)a.out + ((int64_t)sub * a.S + s) * 16 * a.pitch + NT * b * kActRows;
    const int lane = threadIdx.x & 63;
    for (int ch = threadIdx.x >> 6; ch < 16; ch += 4)
        for (int c = lane; c < cols; c += 64) out[(int64_t)ch * a.pitch + c] = turn[ch * P + c];
}

unsigned grid_of(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 20); }
bool rows_of_16_bytes(const void *p, int64_t ld, int dtype) {
    const int eb = dtype == F32 ? 4 : 2;
    return ((uintptr_t)p & 15) == 0 && (ld * eb & 15) == 0;
}

}  // namespace

hipError_t launch_mx4_quantize(const Mx4QuantArgs &a, hipStream_t s) {
    const bool vec = rows_of_16_bytes(a.src, a.ld, a.dtype);
    const unsigned grid = grid_of((int64_t)a.n_rg * mx4_tiles(a.K) * 64);
    if (a.dtype == F32)
        hipLaunchKernelGGL(k_mx4_quantize<F32T>, dim3(grid), dim3(256), 0, s, a, vec);
    else
        hipLaunchKernelGGL(k_mx4_quantize<BF16T>, dim3(grid), dim3(256), 0, s, a, vec);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4DequantArgs &a, hipStream_t s) {
    const bool vec = rows_of_16_bytes(a.dst, a.ld, a.dtype);
    const unsigned grid = grid_of((int64_t)a.w.n_rg * a.w.S * 64);
    if (a.dtype == F32)
        hipLaunchKernelGGL(k_mx4_dequantize<F32T>, dim3(grid), dim3(256), 0, s, a, vec);
    else
        hipLaunchKernelGGL(k_mx4_dequantize<BF16T>, dim3(grid), dim3(256), 0, s, a, vec);
    return hipGetLastError();
}

hipError_t launch_mx4_activations(const Mx4ActArgs &a, hipStream_t s) {
    const bool vec = rows_of_16_bytes(a.x, a.ld, a.dtype);
    const int per_sub = (std::min(a.per, a.n) + kActRows - 1) / kActRows;
    const dim3 grid((unsigned)a.S, (unsigned)((a.n + a.per - 1) / a.per * per_sub));
    if (a.dtype == F32)
        hipLaunchKernelGGL(k_mx4_activations<F32T>, grid, dim3(256), 0, s, a, per_sub, vec);
    else
        hipLaunchKernelGGL(k_mx4_activations<BF16T>, grid, dim3(256), 0, s, a, per_sub, vec);
    return hipGetLastError();
}

}  // namespace swift
