// Products with MXFP4 matrices (format and layout: swift_mx4.h): the projections of a model whose weights are kept so, and the calls that
// are part of no model's pass.
#include <math.h>

#include "swift_device.h"
#include "swift_mv.h"
#include "swift_mx4.h"
#include "swift_mx4_device.h"

namespace swift {

namespace {

// Up to 128 columns: a workgroup per row group, its 8 wavefronts a slice of the super-tiles each.  A column's result is the sum of its slices
// in order, a row's the sum of its terms' in order, so it does not depend on the rows that share the launch.
// (LDS: [8 slices][16 NCB columns][16] sums, [64] scales, [1024] scratch of the norm)
template <int EPI, int NCB>
__global__ __launch_bounds__(512) void k_mx4_mv(Mx4Matrix w, MvArgs a, Mx4Out out, int rg0, int NT, int NC) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int NCP = 16 * NCB;
    constexpr bool kModel = EPI == EPI_QKV || EPI == EPI_RESID || EPI == EPI_SWIGLU;
    float *red = (float *)smem, *rs = red + 8 * NCP * 16, *nscratch = rs + 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const int rg = rg0 + (int)blockIdx.x;
    const int n = (w.S + 7) / 8, s0 = min(wave * n, w.S), s1 = min(s0 + n, w.S);
    if constexpr (kModel && EPI != EPI_RESID) {
        if constexpr (NCB <= 3) {
            mv_norm_finish(a, mv_norm_load(a), rs, nscratch);
        } else if constexpr (NCB == 8) {
            mv_norm64_finish(a, mv_norm64_load(a), rs, nscratch);
        } else {
            mv_norm32_finish(a, mv_norm32_load(a), rs, nscratch);
        }
    }
    f32x4 acc[NCB];
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) acc[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int chunks = kModel ? a.K >> 3 : 16 * w.S;
    for (int s = s0; s < s1; ++s) {
        const size_t piece = (size_t)rg * w.S + s;
        const u32x4 code = *(const u32x4 *)(w.codes + piece * 1024 + lane * 16);
        const float scale = __uint_as_float((uint32_t)w.scales[piece * 64 + lane] << 23);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const bf16x8 av = mx4_decode(code[t], scale);
            const int ch = 16 * s + 4 * kg + t;
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb) {
                u32x4 bv = {0u, 0u, 0u, 0u};
                if (ch < chunks) bv = *(const u32x4 *)((const uint16_t *)a.in_s + ((size_t)ch * NC + min(16 * cb + col, NC - 1)) * 8);
                acc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, bv), acc[cb], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) *(f32x4 *)(red + ((wave * NCP + 16 * cb + col) * 16 + 4 * kg)) = acc[cb];
    __syncthreads();
    auto y = [&](int r, int j) {
        float t[3] = {0.f, 0.f, 0.f};
        for (int i = 0; i < NT; ++i) {
            const float *p = red + (NT * r + i) * 16 + j;
            float v = p[0];
#pragma unroll
            for (int k = 1; k < 8; ++k) v += p[k * NCP * 16];
            t[i] = v;
        }
        return (t[0] + t[1]) + t[2];
    };
    if constexpr (kModel)
        mv_epilogue<EPI>(a, rg, lane, rs, nullptr, y, wave, 8);
    else
        mx4_call_epilogue<EPI>(out, a.R, a.O, rg, tid, 512, y);
}

template <int EPI, int NCB>
hipError_t launch_mx4_mv_t(const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, int rg0, int NT, int NC, hipStream_t s) {
    const size_t lds = (size_t)(8 * 16 * NCB * 16 + 64 + 1024) * 4;  // (at most 70 KB)
    hipError_t e = hipFuncSetAttribute((const void *)k_mx4_mv<EPI, NCB>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mx4_mv<EPI, NCB>), dim3(a.n_rg - rg0), dim3(512), lds, s, w, a, out, rg0, NT, NC);
    return hipGetLastError();
}
template <int EPI>
hipError_t launch_mx4_mv_e(const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, int rg0, int NT, int NC, hipStream_t s) {
    const int ncb = (NC + 15) / 16;
    if (ncb <= 1) return launch_mx4_mv_t<EPI, 1>(w, a, out, rg0, NT, NC, s);
    if (ncb <= 2) return launch_mx4_mv_t<EPI, 2>(w, a, out, rg0, NT, NC, s);
    if (ncb <= 3) return launch_mx4_mv_t<EPI, 3>(w, a, out, rg0, NT, NC, s);
    if (ncb <= 4) return launch_mx4_mv_t<EPI, 4>(w, a, out, rg0, NT, NC, s);
    if (ncb <= 6) return launch_mx4_mv_t<EPI, 6>(w, a, out, rg0, NT, NC, s);
    return launch_mx4_mv_t<EPI, 8>(w, a, out, rg0, NT, NC, s);
}

}  // namespace

hipError_t launch_mx4_mv(int epi, const MvArgs &a, const Mx4Matrix &w, int rg0, hipStream_t s) {
    const bool bulk = (a.RL & kBulkLayout) != 0;
    const int lrows = layout_rows(a.RL), NT = block_terms(a.RL), NC = NT * lrows, ncb = (NC + 15) / 16;
    if (a.R < 1 || a.R > kMaxBlockRows || (a.rp != 16 && a.rp != 64) || a.R > a.rp || a.R > lrows ||
        (bulk ? (lrows != 32 && lrows != 64) : (lrows != a.R || lrows > kMaxRows)) || (a.rp == 16) != (ncb <= 3) || (a.K & 7) != 0 ||
        w.S != mx4_tiles(a.K) || rg0 < 0 || rg0 >= a.n_rg || a.n_rg > w.n_rg || (epi != EPI_RESID && (!a.pss || a.n_pss < 1)))
        return hipErrorInvalidValue;
    switch (epi) {
        case EPI_QKV: return launch_mx4_mv_e<EPI_QKV>(w, a, Mx4Out{}, rg0, NT, NC, s);
        case EPI_RESID: return launch_mx4_mv_e<EPI_RESID>(w, a, Mx4Out{}, rg0, NT, NC, s);
        case EPI_SWIGLU: return launch_mx4_mv_e<EPI_SWIGLU>(w, a, Mx4Out{}, rg0, NT, NC, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_mx4_call(int epi, const Mx4CallArgs &c, hipStream_t s) {
    const int NC = c.n * c.terms;
    if (c.n < 1 || NC > kMx4MaxColumns) return hipErrorInvalidValue;
    MvArgs a{};
    a.R = c.n;
    a.O = c.O;
    a.n_rg = c.w.n_rg;
    a.in_s = c.x;
    if (epi == EPI_LINEAR) return launch_mx4_mv_e<EPI_LINEAR>(c.w, a, c.out, 0, c.terms, NC, s);
    if (epi == EPI_GATED) return launch_mx4_mv_e<EPI_GATED>(c.w, a, c.out, 0, c.terms, NC, s);
    return hipErrorInvalidValue;
}

}  // namespace swift
