// What the blocked matrix products of prompt macro blocks share: the RMSNorm scales of a workgroup's sub-blocks and the epilogues that work
// on accumulators in registers.
#pragma once
#include <math.h>

#include <type_traits>

#include "swift_device.h"
#include "swift_kernels.h"
#include "swift_mv.h"

namespace swift {

constexpr int kNormFloats = 2 * 16 * 64;  // scratch of gemm_norm_scales

// RMSNorm scales of the workgroup's two sub-blocks: rs[64 wn + r].  Thread (wn, q, r4) adds the partials q, q + 16,
// .. of rows 4 r4 .. 4 r4 + 3 of sub-block wn (16 loads of 16 bytes in flight at a time); then one thread per row
// adds the sixteen sums in order.  The first 256 partials are requested ahead of the ring's first stages, so that they do not queue
// behind 140 KB of tiles, and added up once those are on their way, where registers allow (kLateNorm; else before); the scales are read by
// the epilogue only, so no barrier here waits for more than LDS.
struct GemmNorm {
    f32x4 v[16];
};
__device__ inline GemmNorm gemm_norm_load(const MvArgs &a, const MacroArgs &ma, int sub0, int p0 = 0) {
    const int tid = threadIdx.x, q = (tid >> 4) & 15;
    const float *p = a.pss + (size_t)min(sub0 + (tid >> 8), ma.S - 1) * ma.pss + 4 * (tid & 15);
    GemmNorm n;
#pragma unroll
    for (int u = 0; u < 16; ++u) n.v[u] = *(const f32x4 *)(p + (size_t)min(p0 + q + 16 * u, a.n_pss - 1) * a.rp);
    return n;
}
__device__ inline f32x4 gemm_norm_sum(const MvArgs &a, const MacroArgs &ma, int sub0, const GemmNorm &first) {
    const int q = (threadIdx.x >> 4) & 15;
    f32x4 ss = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](int p0, const GemmNorm &n) {
#pragma unroll
        for (int u = 0; u < 16; ++u) ss += p0 + q + 16 * u < a.n_pss ? n.v[u] : f32x4{0.f, 0.f, 0.f, 0.f};
    };
    add(0, first);
    for (int p0 = 256; p0 < a.n_pss; p0 += 256) add(p0, gemm_norm_load(a, ma, sub0, p0));
    return ss;
}
__device__ inline void gemm_norm_scales(const MvArgs &a, const f32x4 &ss, float *rs, float *scratch) {
    const int tid = threadIdx.x, r4 = tid & 15, q = (tid >> 4) & 15, wn = tid >> 8;
    *(f32x4 *)(scratch + (wn * 16 + q) * 64 + 4 * r4) = ss;
    lds_barrier();
    if (tid < 128) {
        const int w2 = tid >> 6, r2 = tid & 63;
        float sum = 0.f;
#pragma unroll
        for (int q2 = 0; q2 < 16; ++q2) sum += scratch[(w2 * 16 + q2) * 64 + r2];
        rs[tid] = 1.0f / sqrtf(sum / (float)a.norm_dim + a.eps);
    }
}

// ------------------------------------------------------------------------------------------
// epilogue
// ------------------------------------------------------------------------------------------
// It works on the accumulators where they are: a wavefront's 4 accumulator tiles of a row group hold column 16 cb + col
// = 2 r + term in lane column col, tile rows 4 kg .. 4 kg + 3 in the lane's four registers.  The two terms of a block
// row sit in neighbouring lanes; the even lane keeps the even column blocks, the odd lane the odd ones, so that a lane
// ends up with two block rows r(c) = r0 + 16 c + 8 (col & 1) + col / 2, c = 0, 1 (r0: first row of the wavefront's half of
// the sub-block), and four consecutive tile rows of each: 16-byte reads and writes of everything that is laid out along the rows of W, and no trip through LDS.  (The
// block kernel's epilogue, which this replaces here, walks a row group in sixteen dependent rounds of a load, a few
// LDS reads and 2-byte stores: about 10 us per row group and wavefront, 20-43 us per workgroup, a third of a 512-row
// launch; now 4-9 us.)
__device__ inline float dpp_xor1(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
}
__device__ inline int gemm_row(int c, int col) { return 16 * c + 8 * (col & 1) + (col >> 1); }  // within the wavefront's 32 rows
__device__ inline void fold_terms(const f32x4 (&acc)[4], int col, f32x4 (&y)[2]) {
    const bool odd = col & 1;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float own = odd ? acc[2 * c + 1][i] : acc[2 * c][i], other = odd ? acc[2 * c][i] : acc[2 * c + 1][i];
            y[c][i] = own + dpp_xor1(other);
        }
}
// Exchanges the upper 32 lanes of a with the lower ones of b.
__device__ inline void swap32(float &a, float &b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
// The two-term split of the four values of lanes kg, kg ^ 1 (values 4 (kg & 1) .. of eight), to unit
// [chunk][128 columns][8]: columns 2 r and 2 r + 1.
__device__ inline void store_split(uint16_t *out_s, int chunk, int r, int kg, bool ok, const f32x4 &v) {
    uint32_t h[4], m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = f32_to_bf16_rne_finite(v[i]);
        m[i] = f32_to_bf16_rne_finite(v[i] - __uint_as_float(h[i] << 16));
    }
    const u32x4 u = join8(pack2(h[0], h[1]), pack2(h[2], h[3]), pack2(m[0], m[1]), pack2(m[2], m[3]));
    if (ok) *(u32x4 *)(out_s + ((size_t)chunk * 128 + 2 * r + (kg & 1)) * 8) = u;
}

// x += y for RGW row groups from rg0 and rows r0 .. r0 + 31: the residual values and gains of up to four of them are
// requested together.  y(g, out): finished sums of row group g.
template <int RGW, typename YF>
__device__ inline void gemm_resid(const MvArgs &a, int rg0, int r0, int lane, YF y) {
    const int col = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int g0 = 0; g0 < RGW; g0 += 4) {
        constexpr int G = RGW < 4 ? RGW : 4;
        f32x4 x[G][2], gain[G];
#pragma unroll
        for (int g = 0; g < G && g0 + g < RGW; ++g) {
            const int row = 16 * (rg0 + g0 + g) + 4 * kg;
            const bool in = row < a.O;  // (O is a multiple of 8: a lane's four rows are all real or all padding)
            gain[g] = in ? *(const f32x4 *)(a.gain_next + row) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = r0 + gemm_row(c, col);
                x[g][c] = in && r < a.R ? *(const f32x4 *)(a.out_f32 + (size_t)r * a.ld_out + row) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
#pragma unroll
        for (int g = 0; g < G && g0 + g < RGW; ++g) {
            const int rg = rg0 + g0 + g, row = 16 * rg + 4 * kg;
            if (rg >= a.n_rg) return;  // (wavefront-uniform)
            const bool in = row < a.O;
            f32x4 v[2];
            y(g0 + g, v);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = r0 + gemm_row(c, col);
                const bool ok = in && r < a.R;
                const f32x4 xn = x[g][c] + v[c];
                if (ok) *(f32x4 *)(a.out_f32 + (size_t)r * a.ld_out + row) = xn;
                store_split(a.out_s, 2 * rg + (kg >> 1), r, kg, ok, xn * gain[g]);
                float ss = in ? (xn[0] * xn[0] + xn[1] * xn[1]) + (xn[2] * xn[2] + xn[3] * xn[3]) : 0.f;
                ss = column_reduce(ss, [](float x, float y) { return x + y; });
                if (kg == 0 && r < a.R) a.pss_out[(size_t)rg * a.rp + r] = ss;
            }
        }
    }
}

// A lane's two block rows paired up: the first eight tile rows (gate, or the first half of rotary pairs) of c =
// kg >> 1 end up in lo, the other eight of the same block row in hi (tile rows 4 (kg & 1) .. of each), scaled.
__device__ inline void pair_halves(const f32x4 (&v)[2], const float (&sc)[2], f32x4 &lo, f32x4 &hi) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = v[0][i] * sc[0], y = v[1][i] * sc[1];
        swap32(x, y);
        lo[i] = x;
        hi[i] = y;
    }
}

__device__ inline void gemm_swiglu(const MvArgs &a, int rg, int r0, int lane, const float (&sc)[2], const f32x4 (&v)[2]) {
    const int col = lane & 15, kg = lane >> 4;
    f32x4 ga, up, h;
    pair_halves(v, sc, ga, up);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = ga[i] / (1.0f + expf(-ga[i])) * up[i];
    const int r = r0 + gemm_row(kg >> 1, col);
    store_split(a.out_s, rg, r, kg, r < a.R && 16 * rg < a.O, h);
}

// Queries to fp32 rows, keys to their slots, values to the grouped layout: there, eight consecutive slots of an element
// are one 16-byte unit, so the values cross the lanes through a wavefront's own 1.3 KB of LDS (vsh).
template <int RGW, typename YF>
__device__ inline void gemm_qkv(const MvArgs &a, int rg0, int r0, int lane, const float (&sc)[2], uint16_t *vsh, YF y) {
    constexpr int VP = 32 + 8;  // pitch of an element's slots in vsh
    const int col = lane & 15, kg = lane >> 4;
    const int d = a.head_dim, half = d >> 1, gph = half >> 3, nq = a.n_q_heads, nkv = a.n_kv_heads;
    const int rl = gemm_row(kg >> 1, col), r = r0 + rl, pos = a.pos0 + r;  // the lane's block row, once paired up
    const bool ok = r < a.R;
    f32x4 cs[RGW], sn[RGW];
#pragma unroll
    for (int g = 0; g < RGW; ++g) {
        const int rg = min(rg0 + g, a.n_rg - 1), i0 = 8 * (rg % gph) + 4 * (kg & 1);
        cs[g] = *(const f32x4 *)(a.cos_tab + (size_t)(a.pos0 + min(r, a.R - 1)) * half + i0);
        sn[g] = *(const f32x4 *)(a.sin_tab + (size_t)(a.pos0 + min(r, a.R - 1)) * half + i0);
    }
#pragma unroll
    for (int g = 0; g < RGW; ++g) {
        const int rg = rg0 + g;
        if (rg >= a.n_rg) break;  // (wavefront-uniform)
        const int hl = rg / gph, hh = a.head0 + hl, e0 = 8 * (rg - hl * gph);  // head; first element of the row group's eight pairs
        f32x4 v[2], ya, yb;
        y(g, v);
        pair_halves(v, sc, ya, yb);
        if (hh < nq + nkv) {
            const f32x4 qa = ya * cs[g] - yb * sn[g], qb = yb * cs[g] + ya * sn[g];
            if (hh < nq) {
                float *qp = a.out_f32 + (size_t)r * a.ld_out + hh * d + e0 + 4 * (kg & 1);
                if (ok) {
                    *(f32x4 *)qp = qa;
                    *(f32x4 *)(qp + half) = qb;
                }
                continue;
            }
            ya = qa;
            yb = qb;
        }
        uint32_t ha[4], hb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ha[i] = f32_to_bf16_rne(ya[i]);
            hb[i] = f32_to_bf16_rne(yb[i]);
        }
        if (hh < nq + nkv || a.nb32 <= 0) {
            const int head = hh < nq + nkv ? hh - nq : hh - nq - nkv;
            uint16_t *plane = (uint16_t *)(hh < nq + nkv ? a.kcache : a.vcache);
            const u32x4 u = join8(pack2(ha[0], ha[1]), pack2(ha[2], ha[3]), pack2(hb[0], hb[1]), pack2(hb[2], hb[3]));
            if (ok) *(u32x4 *)(plane + ((size_t)head * a.max_seq + pos) * d + e0 + (kg & 1) * half) = u;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vsh[(4 * (kg & 1) + i) * VP + rl] = (uint16_t)ha[i];
                vsh[(8 + 4 * (kg & 1) + i) * VP + rl] = (uint16_t)hb[i];
            }
            // (one wavefront's LDS instructions are carried out in order: only the compiler has to keep it)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const int e = lane & 15, elem = e0 + (e & 7) + (e >> 3) * half;
            const int u8 = 8 * (lane >> 4), ru = r0 + u8;  // eight slots from block row ru on
            const u32x4 w = *(const u32x4 *)(vsh + e * VP + u8);
            uint16_t *vp = (uint16_t *)a.vcache;
            if ((a.pos0 & 7) == 0 && ru + 8 <= a.R) {
                *(u32x4 *)(vp + kv_vt_index(hh - nq - nkv, a.nb32, d, a.pos0 + ru, elem)) = w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ru + i < a.R)
                        vp[kv_vt_index(hh - nq - nkv, a.nb32, d, a.pos0 + ru + i, elem)] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

}  // namespace swift
