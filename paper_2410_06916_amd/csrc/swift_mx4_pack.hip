// MXFP4 matrices: numbers to packed blocks and back, and activations to the B operand's layout (formats: swift_mx4.h).
#include <algorithm>

#include "swift_device.h"
#include "swift_mx4.h"
#include "swift_mx4_device.h"

namespace swift {

namespace {

// Both ways a wavefront has four rows by 128 k, so that rows are read and written in pieces of 16 lanes x 16 bytes next to each other (quantising,
// four lanes share a block and a lane has eight elements, a word of codes); a workgroup covers a piece (16 rows x 128 k) and walks kAhead of them, whose
// loads go out together.  What bounds both is memory.  (A lane per block reads and writes 64 lines an instruction: the 7B gate and up pair
// there and back 130 us; so 74, 5.5 TB/s.)
constexpr int kAhead = 4;
struct PieceLane {
    int j, kg, w;  // tile row, block, word
};
__device__ inline PieceLane piece_lane() {
    const int t = threadIdx.x;
    return {t >> 4, (t >> 2) & 3, t & 3};
}
// The largest over the four lanes of a block.
__device__ inline uint32_t block_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
}

// Row of the matrix in tile row j of row group rg.
__device__ inline int tile_row(int mode, int d, int rg, int j) {
    if (mode == TILE_PLAIN) return 16 * rg + j;
    if (mode == TILE_GATEUP) return 8 * rg + (j & 7);
    const int gph = d >> 4, head = rg / gph, g = rg - head * gph;
    return head * d + 8 * g + (j & 7) + (j >= 8 ? d >> 1 : 0);
}

// The scale's exponent is that of the largest magnitude less two (its floor(log2) against the four of the largest element's binade), at least
// -127; the conversion instruction divides by the scale, rounds to the nearest element, ties to the even code, and saturates at 6,
// subnormals included.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_quantize(Mx4QuantArgs a, bool vec) {
    const int S = mx4_tiles(a.K), rg = blockIdx.y, s0 = blockIdx.x * kAhead;
    const PieceLane l = piece_lane();
    const bool up = a.mode == TILE_GATEUP && l.j >= 8;
    if (a.mode == TILE_GATEUP && !(up ? a.up : a.src)) return;  // (that half comes another time; whole blocks leave)
    const int row = tile_row(a.mode, a.head_dim, rg, l.j), kl = kMx4Block * l.kg + 8 * l.w;
    const auto *src = (const typename T::elem *)(up ? a.up : a.src) + (int64_t)row * (up ? a.ld_up : a.ld);
    const int K = row < a.src_rows ? a.K : 0;  // (rows and k past the matrix: zeros)
    float v[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) mx4_load8<T>(src, kMx4Tile * (s0 + i) + kl, K, vec, v[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        if (s0 + i >= S) break;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[i][k]) & 0x7fffffffu);  // (NaNs above infinity above numbers)
        uint32_t e = block_max(top) >> 23, q = 0;
        if (e != 255) {
            e = e > 2 ? e - 2 : 0;
            const float scale = __uint_as_float(e << 23);  // (the instructions read its exponent field only: 0 is 2^-127)
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][0], v[i][1], scale, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][2], v[i][3], scale, 1);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][4], v[i][5], scale, 2);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[i][6], v[i][7], scale, 3);
        }
        const int64_t piece = (int64_t)rg * S + s0 + i;
        ((uint32_t *)a.codes)[piece * 256 + (16 * l.kg + l.j) * 4 + l.w] = q;
        if (l.w == 0) a.scales[piece * 64 + 16 * l.kg + l.j] = (uint8_t)e;
    }
}

// A lane writes 16 bytes at a time, next to its neighbours': in fp32 four elements, half a word of codes, of either half of the piece.
// fp32, 13B down projection, us: eight elements in a row as two stores of every other 16 bytes 84; so 73; past the caches, which such results
// do not fit, 49 (6.6 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_dequantize(Mx4DequantArgs a, bool vec) {
    constexpr int V = T::VEC, N = 8 / V;  // elements of a store, stores of a piece
    const int S = a.w.S, rg = blockIdx.y, s0 = blockIdx.x * kAhead, j = threadIdx.x >> 4, l = threadIdx.x & 15;
    const int row = a.row0 + tile_row(a.mode, 0, rg, j);
    if (row >= a.rows) return;
    auto *dst = (typename T::elem *)a.dst + (int64_t)(a.mode == TILE_GATEUP && j >= 8 ? row + a.rows : row) * a.ld;
    uint32_t code[kAhead][N], e[kAhead][N];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const int64_t piece = (int64_t)rg * S + min(s0 + i, S - 1);
            const int k = (16 * h + l) * V, at = 16 * (k / kMx4Block) + j;  // of the super-tile; the block's place in the piece
            const uint8_t *c = a.w.codes + piece * 1024 + at * 16 + k % kMx4Block / 2;
            code[i][h] = V == 8 ? *(const uint32_t *)c : *(const uint16_t *)c;
            e[i][h] = a.w.scales[piece * 64 + at];
        }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        if (s0 + i >= S) break;
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const int k = kMx4Tile * (s0 + i) + (16 * h + l) * V;
            // (every value is a bf16 number, subnormal ones included: nothing is rounded)
            const u32x4 y = __builtin_bit_cast(u32x4, mx4_decode(code[i][h], __uint_as_float(e[i][h] << 23)));
            auto value = [&](int u) { return __uint_as_float(u & 1 ? y[u / 2] & 0xffff0000u : y[u / 2] << 16); };
            if (vec && k + V <= a.K) {
                if constexpr (V == 8)
                    __builtin_nontemporal_store(y, (u32x4 *)(dst + k));
                else
                    __builtin_nontemporal_store(f32x4{value(0), value(1), value(2), value(3)}, (f32x4 *)(dst + k));
            } else {
#pragma unroll
                for (int u = 0; u < V; ++u)
                    if (k + u < a.K) T::store1(dst + k + u, value(u));
            }
        }
    }
}

// A workgroup turns 64 rows (at most) of a sub-block by 16 chunks through LDS: rows are read 128 k at a time, columns are written a KB at a
// time.  (A thread per chunk that writes where its chunk goes: 512 rows of 4096 bf16 7.5 us; so 4.2,
// of which a launch is 1.7.)
constexpr int kActRows = 64;
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_activations(Mx4ActArgs a, int blocks_of_sub, bool vec) {
    constexpr int NT = T::VEC == 8 ? 1 : 3, P = kActRows * NT + 1;
    __shared__ u32x4 turn[16 * P];
    const int s = blockIdx.x, sub = blockIdx.y / blocks_of_sub, b = blockIdx.y - sub * blocks_of_sub;
    const int r0 = sub * a.per + b * kActRows, rows = min(kActRows, min(a.per - b * kActRows, a.n - r0));
    if (rows <= 0) return;
    float v[4][8];  // (all loads together)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = (threadIdx.x >> 4) + 16 * j, k0 = kMx4Tile * s + 8 * (threadIdx.x & 15);
        mx4_load8<T>((const typename T::elem *)a.x + (int64_t)(r0 + r) * a.ld, k0, r < rows ? a.K : 0, vec, v[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = (threadIdx.x >> 4) + 16 * j, ch = threadIdx.x & 15;
        if (r >= rows) break;
        u32x4 t[3];
        if constexpr (NT == 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) t[0][i] = (__float_as_uint(v[j][2 * i]) >> 16) | (__float_as_uint(v[j][2 * i + 1]) & 0xffff0000u);
        } else {
            mx4_split8(v[j], t);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) turn[ch * P + NT * r + i] = t[i];
    }
    __syncthreads();
    const int cols = NT * rows;
    u32x4 *out = (u32x4 *)a.out + ((int64_t)sub * a.S + s) * 16 * a.pitch + NT * b * kActRows;
    const int lane = threadIdx.x & 63;
    for (int ch = threadIdx.x >> 6; ch < 16; ch += 4)
        for (int c = lane; c < cols; c += 64) out[(int64_t)ch * a.pitch + c] = turn[ch * P + c];
}

bool rows_of_16_bytes(const void *p, int64_t ld, int dtype) {
    const int eb = dtype == F32 ? 4 : 2;
    return ((uintptr_t)p & 15) == 0 && (ld * eb & 15) == 0;
}

}  // namespace

// Row groups of one launch (the grid's second dimension).
constexpr int kMaxRowGroups = 65535;

hipError_t launch_mx4_quantize(const Mx4QuantArgs &args, hipStream_t s) {
    const bool vec = (!args.src || rows_of_16_bytes(args.src, args.ld, args.dtype)) && (!args.up || rows_of_16_bytes(args.up, args.ld_up, args.dtype));
    const int S = mx4_tiles(args.K), eb = args.dtype == F32 ? 4 : 2;
    if (args.mode == TILE_PAIR && args.n_rg > kMaxRowGroups) return hipErrorInvalidValue;
    for (int rg0 = 0; rg0 < args.n_rg; rg0 += kMaxRowGroups) {
        Mx4QuantArgs a = args;
        const int64_t skipped = (int64_t)rg0 * (a.mode == TILE_GATEUP ? 8 : 16);  // rows
        if (a.src) a.src = (const char *)a.src + skipped * a.ld * eb;
        if (a.up) a.up = (const char *)a.up + skipped * a.ld_up * eb;
        a.src_rows -= (int)skipped;
        a.codes += (int64_t)rg0 * S * 1024;
        a.scales += (int64_t)rg0 * S * 64;
        const dim3 grid((unsigned)((S + kAhead - 1) / kAhead), (unsigned)std::min(kMaxRowGroups, a.n_rg - rg0));
        if (a.dtype == F32)
            hipLaunchKernelGGL(k_mx4_quantize<F32T>, grid, dim3(256), 0, s, a, vec);
        else
            hipLaunchKernelGGL(k_mx4_quantize<BF16T>, grid, dim3(256), 0, s, a, vec);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_mx4_dequantize(const Mx4DequantArgs &args, hipStream_t s) {
    const bool vec = rows_of_16_bytes(args.dst, args.ld, args.dtype);
    for (int rg0 = 0; rg0 < args.w.n_rg; rg0 += kMaxRowGroups) {
        Mx4DequantArgs a = args;
        a.w.codes += (int64_t)rg0 * a.w.S * 1024;
        a.w.scales += (int64_t)rg0 * a.w.S * 64;
        a.row0 = rg0 * (a.mode == TILE_GATEUP ? 8 : 16);
        const dim3 grid((unsigned)((a.w.S + kAhead - 1) / kAhead), (unsigned)std::min(kMaxRowGroups, args.w.n_rg - rg0));
        if (a.dtype == F32)
            hipLaunchKernelGGL(k_mx4_dequantize<F32T>, grid, dim3(256), 0, s, a, vec);
        else
            hipLaunchKernelGGL(k_mx4_dequantize<BF16T>, grid, dim3(256), 0, s, a, vec);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
