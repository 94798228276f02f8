// Epilogue of the tiled projection kernels, and the RMSNorm scales that it applies.
#pragma once
#include <math.h>

#include "swift_device.h"
#include "swift_kernels.h"

namespace swift {

// Values in the grouped layout (kv_vt_index) are written two bytes at a time into 128-byte lines that the
// pass fills only partly, and such a store completes only once the rest of the line has been fetched.  The
// projection kernel therefore touches the lines its epilogue will write while the weights stream: this is where lane
// (block row r, half) of the calling wavefront reads one word, in the line that holds elements 8 g .. 8 g + 7 (+ d/2) of row r's
// slot, or nullptr: rg is no row group of the value part of the fused q|k|v matrix.  The word is never used.
__device__ inline const uint32_t *mv_value_line(const MvArgs &a, int rg, int lane) {
    const int d = a.head_dim, half = d >> 1, lg = __builtin_ctz(half >> 3);  // (16 .. 128: a power of two)
    const int hh = rg >> lg, head = hh - a.n_q_heads - a.n_kv_heads;
    const int r = lane >> 1;
    if (a.nb32 <= 0 || head < 0 || head >= a.n_kv_heads || r >= a.R) return nullptr;
    const int i = 8 * (rg - (hh << lg)) + (lane & 1) * half;
    return (const uint32_t *)((const uint16_t *)a.vcache + (kv_vt_index(head, a.nb32, d, a.pos0 + r, i) & ~(size_t)1));
}
// What follows the dot products of one 16-row group, run by one whole wavefront.
// Y(r, j): finished dot product of block row r and tile row j (before the norm scale).
// rot: optional LDS copy of the rotary rows (k_mv1), [R][d/2] cosines, then sines at mv1_rot_pitch; nullptr = read the tables.
// Several wavefronts may share a row group: wavefront it0 of it_step takes every it_step-th pass of 64 results.
// X: EPI_RESID's residual values, requested ahead of time (mv_residuals), or NoResiduals.
struct NoResiduals {
    static constexpr int N = 0;
};
template <int XN>
struct Residuals {
    static constexpr int N = XN;
    float x[XN], gain;
};
// The residual values that the first XN passes of a wavefront's share of a row group's epilogue add to, and the gain of the lane's row.
template <int XN>
__device__ inline Residuals<XN> mv_residuals(const MvArgs &a, int rg, int lane, int it0 = 0, int it_step = 1) {
    Residuals<XN> X;
    const int row = min(16 * rg + (lane & 15), a.O - 1);
    X.gain = a.gain_next[row];
#pragma unroll
    for (int k = 0; k < XN; ++k) X.x[k] = a.out_f32[(size_t)min(4 * (it0 + k * it_step) + (lane >> 4), a.R - 1) * a.ld_out + row];
    return X;
}
template <int EPI, typename YF, typename XT = NoResiduals>
__device__ inline void mv_epilogue(const MvArgs &a, int rg, int lane, const float *rs, const float *rot, YF Y, int it0 = 0,
                                   int it_step = 1, const XT &X = XT()) {
    const int R = a.R, NT = block_terms(a.RL), NC = NT * layout_rows(a.RL);  // NC: column pitch of the split outputs
    if (EPI == EPI_RESID || EPI == EPI_LOGITS) {
        const int iters = (16 * R + 63) >> 6;
        const int j = lane & 15, row = 16 * rg + j;
        auto pass = [&](int it, float x, float gain) {
            const int r = 4 * it + (lane >> 4);
            const bool ok = r < R && row < a.O;
            if (EPI == EPI_LOGITS) {
                if (ok) a.out_f32[(size_t)r * a.ld_out + row] = Y(r, j) * rs[r];
            } else {
                float xn = 0.f;
                if (ok) {
                    xn = x + Y(r, j);
                    a.out_f32[(size_t)r * a.ld_out + row] = xn;
                    uint16_t hi, mid, lo;
                    split3(xn, gain, hi, mid, lo);
                    uint16_t *p = a.out_s + ((size_t)(row >> 3) * NC + NT * r) * 8 + (row & 7);
                    p[0] = hi;
                    p[8] = mid;
                    if (NT == 3) p[16] = lo;
                }
                const float ss = row_sum_of_squares(xn);
                if (r < R && j == 0) a.pss_out[(size_t)rg * a.rp + r] = ss;
            }
        };
        if constexpr (EPI == EPI_RESID && XT::N > 0) {
#pragma unroll
            for (int k = 0; k < XT::N; ++k)
                if (it0 + k * it_step < iters) pass(it0 + k * it_step, X.x[k], X.gain);
        }
        for (int it = it0 + XT::N * it_step; it < iters; it += it_step) {
            float x = 0.f, gain = 0.f;
            if (EPI == EPI_RESID && row < a.O) {
                x = a.out_f32[(size_t)min(4 * it + (lane >> 4), R - 1) * a.ld_out + row];
                gain = a.gain_next[row];
            }
            pass(it, x, gain);
        }
    } else {
        const int iters = (8 * R + 63) >> 6;
        for (int it = it0; it < iters; it += it_step) {
            const int idx = it * 64 + lane;
            const int r = idx >> 3, j = idx & 7;
            if (r >= R) continue;
            const float sc = rs[r];
            const float ya = Y(r, j) * sc, yb = Y(r, j + 8) * sc;
            if (EPI == EPI_SWIGLU) {
                if (2 * (8 * rg + j) < a.O) {
                    uint16_t hi, mid, lo;
                    split3(ya / (1.0f + expf(-ya)), yb, hi, mid, lo);
                    uint16_t *p = a.out_s + ((size_t)rg * NC + NT * r) * 8 + j;
                    p[0] = hi;
                    p[8] = mid;
                    if (NT == 3) p[16] = lo;
                }
            } else {
                const int d = a.head_dim, half = d >> 1, lg = __builtin_ctz(half >> 3);
                const int hh = rg >> lg, i = 8 * (rg - (hh << lg)) + j;
                const int nq = a.n_q_heads, nkv = a.n_kv_heads, pos = a.pos0 + r, rpos = mv_rope_pos(a, r);
                if (hh < nq + nkv) {
                    const float c = rot ? rot[r * half + i] : a.cos_tab[(size_t)rpos * half + i];
                    const float s = rot ? rot[((R * half + 63) & ~63) + r * half + i] : a.sin_tab[(size_t)rpos * half + i];
                    const float qa = ya * c - yb * s, qb = yb * c + ya * s;
                    if (hh < nq) {
                        float *qp = a.out_f32 + (size_t)r * a.ld_out + hh * d + i;
                        qp[0] = qa;
                        qp[half] = qb;
                        if (a.q_s) {
                            uint16_t *qs = a.q_s + ((size_t)(r * nq + hh) * 2) * d + i;
                            const uint32_t ha = f32_to_bf16_rne_finite(qa), hb = f32_to_bf16_rne_finite(qb);
                            qs[0] = (uint16_t)ha;
                            qs[half] = (uint16_t)hb;
                            qs[d] = (uint16_t)f32_to_bf16_rne_finite(qa - __uint_as_float(ha << 16));
                            qs[d + half] = (uint16_t)f32_to_bf16_rne_finite(qb - __uint_as_float(hb << 16));
                        }
                    } else {
                        uint16_t *kc = (uint16_t *)a.kcache + ((size_t)(hh - nq) * a.max_seq + pos) * d + i;
                        kc[0] = f32_to_bf16_rne(qa);
                        kc[half] = f32_to_bf16_rne(qb);
                    }
                } else if (a.nb32 > 0) {  // values in groups of eight slots
                    uint16_t *vc = (uint16_t *)a.vcache + kv_vt_index(hh - nq - nkv, a.nb32, d, pos, i);
                    vc[0] = f32_to_bf16_rne(ya);
                    vc[half * 8] = f32_to_bf16_rne(yb);
                } else {
                    uint16_t *vc = (uint16_t *)a.vcache + ((size_t)(hh - nq - nkv) * a.max_seq + pos) * d + i;
                    vc[0] = f32_to_bf16_rne(ya);
                    vc[half] = f32_to_bf16_rne(yb);
                }
            }
        }
    }
}

// RMSNorm scale per block row from the producer's partial sums of squares.  A kernel requests the first 256 partials of its rows
// (hidden <= 4096: all of them) ahead of its weights and adds them up once the weights are on their way: no branches
// and no use of a loaded value in between (a partial past the last is the last one again, left out of the sum later), since a
// wait there would hold the weights up.  The summation order is fixed.  One barrier, which orders LDS only, before the final sums.
//
// Up to 16 rows (row pitch 16): thread (q = t / 16, row r = t % 16) adds the partials q + 32 u in order of u, then 16 threads
// add the 32 sums in order.
struct NormPart {
    float v[8];
};
__device__ inline NormPart mv_norm_load(const MvArgs &a, int p0 = 0) {
    NormPart np;
    const uint32_t at = threadIdx.x + 16 * p0, end = 16 * a.n_pss - 1;  // partial p of row r is word 16 p + r
#pragma unroll
    for (int u = 0; u < 8; ++u) np.v[u] = *(const float *)((const char *)a.pss + 4 * min(at + 512 * u, end));
    return np;
}
__device__ inline void mv_norm_finish(const MvArgs &a, const NormPart &np, float *rs /* LDS [16] */, float *scratch /* LDS [512] */) {
    const int tid = threadIdx.x, q = tid >> 4;
    float ss = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) ss += q + 32 * u < a.n_pss ? np.v[u] : 0.f;
    for (int p0 = 256; p0 < a.n_pss; p0 += 256) {
        const NormPart more = mv_norm_load(a, p0);
#pragma unroll
        for (int u = 0; u < 8; ++u) ss += p0 + q + 32 * u < a.n_pss ? more.v[u] : 0.f;
    }
    scratch[tid] = ss;
    lds_barrier();
    if (tid < 16) {
        float t = 0.f;
#pragma unroll
        for (int q2 = 0; q2 < 32; ++q2) t += scratch[q2 * 16 + tid];
        rs[tid] = 1.0f / sqrtf(t / (float)a.norm_dim + a.eps);
    }
    // (no barrier here: the scales are read by the epilogue only, and every caller has a barrier between
    // this point and its epilogue)
}

// The same for exact layouts of 17..32 rows (row pitch 64), in the same order -- a row's scale must not depend on the rows it
// shares a pass with: thread (row r, q) adds the partials q + 32 u and q + 16 + 32 u as two sums; then 32 threads add the 32 sums
// in order.
struct NormPart32 {
    float v[2][8];
};
__device__ inline NormPart32 mv_norm32_load(const MvArgs &a, int p0 = 0) {
    NormPart32 np;
    const uint32_t r = threadIdx.x & 31, at = 64 * (p0 + (threadIdx.x >> 5)) + r, end = 64 * (a.n_pss - 1) + r;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int u = 0; u < 8; ++u) np.v[half][u] = *(const float *)((const char *)a.pss + 4 * min(at + 64 * (16 * half + 32 * u), end));
    return np;
}
__device__ inline void mv_norm32_finish(const MvArgs &a, const NormPart32 &np, float *rs /* LDS [32] */, float *scratch /* LDS [1024] */) {
    const int tid = threadIdx.x, r = tid & 31, q0 = tid >> 5;
    float ss[2] = {0.f, 0.f};
    auto add = [&](int p0, const NormPart32 &n) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < 8; ++u) ss[half] += p0 + q0 + 16 * half + 32 * u < a.n_pss ? n.v[half][u] : 0.f;
    };
    add(0, np);
    for (int p0 = 256; p0 < a.n_pss; p0 += 256) add(p0, mv_norm32_load(a, p0));
    scratch[q0 * 32 + r] = ss[0];
    scratch[(q0 + 16) * 32 + r] = ss[1];
    lds_barrier();
    if (tid < 32) {
        float t = 0.f;
#pragma unroll
        for (int q2 = 0; q2 < 32; ++q2) t += scratch[q2 * 32 + tid];
        rs[tid] = 1.0f / sqrtf(t / (float)a.norm_dim + a.eps);
    }
}

// The same for bulk layouts of 64 rows: thread = (partial p mod 8, row r), then 64 threads add the 8 per-thread sums in order.
struct NormPart64 {
    float v[32];
};
__device__ inline NormPart64 mv_norm64_load(const MvArgs &a, int p0 = 0) {
    NormPart64 np;
    const uint32_t at = threadIdx.x + 64 * p0, end = 64 * (a.n_pss - 1) + (threadIdx.x & 63);  // partial p of row r is word 64 p + r
#pragma unroll
    for (int u = 0; u < 32; ++u) np.v[u] = *(const float *)((const char *)a.pss + 4 * min(at + 512 * u, end));
    return np;
}
__device__ inline void mv_norm64_finish(const MvArgs &a, const NormPart64 &np, float *rs /* LDS [64] */, float *scratch /* LDS [512] */) {
    const int tid = threadIdx.x, q = tid >> 6;
    float ss = 0.f;
    auto add = [&](int p0, const NormPart64 &n) {
#pragma unroll
        for (int u = 0; u < 32; ++u) ss += p0 + q + 8 * u < a.n_pss ? n.v[u] : 0.f;
    };
    add(0, np);
    for (int p0 = 256; p0 < a.n_pss; p0 += 256) add(p0, mv_norm64_load(a, p0));
    scratch[tid] = ss;
    lds_barrier();
    if (tid < 64) {
        float t = 0.f;
#pragma unroll
        for (int q2 = 0; q2 < 8; ++q2) t += scratch[q2 * 64 + tid];
        rs[tid] = 1.0f / sqrtf(t / (float)a.norm_dim + a.eps);
    }
}

}  // namespace swift
