// Products with MXFP4 matrices (format and layout: swift_mx4.h): the projections of a model whose weights are kept so, and the calls that
// are part of no model's pass.
#include <math.h>

#include "swift_device.h"
#include "swift_mv.h"
#include "swift_mx4.h"
#include "swift_mx4_device.h"

namespace swift {

namespace {

// Few rows: the weight stream is what bounds these launches, and, where the matrix is small, what a launch costs before and after it.
//
// A workgroup's 8 wavefronts each own an eighth of the super-tiles (a slice) of RG row groups at a time, all columns; their sums meet in LDS,
// in the order of the slices, a row's terms after that: a row's result does not depend on the rows that share the launch, nor
// on RG.  A slice is a buffer: past its end loads read nothing.
// ONE: the window of NA super-tiles holds the whole slice and a workgroup has one round of row groups, so nothing is asked for twice;
// several workgroups share a compute unit and overlap each other's ends.  Else rounds roll on in one launch: the loads of the next
// round's first super-tiles go out as the registers of the last ones' come free.
// B (up to 16 columns: SRC 1 and 2): every wavefront copies its own slice into LDS ahead of the weights, as it lies (bf16), or splits it there
// (fp32 rows of a call); no barrier, and no registers beside those of the weights' window.  More columns (SRC 0): B from L2 into
// registers, a window of NBQ quarters.
enum Mx4Source : int { kRegisters = 0, kLds = 1, kLdsSplit = 2 };
struct Mx4MvRest {
    MvArgs a;
    Mx4Out out;
    int NT;
    // kLds: lines of b_bytes bytes, line_pitch bytes apart in memory, copied one after the other; kLdsSplit: rows, ld_x elements apart
    int lines;
    uint32_t line_pitch;
    const float *x32;
    int64_t ld_x;
    int K;
};
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past every buffer: the load reads nothing and gives zeros
constexpr int kNonTemporal = 2;
template <int NCB, int RG>
constexpr bool kMx4TwoBuffers = 2 * 8 * RG * 16 * NCB * 64 <= 64 * 1024;

template <int EPI, int NCB, int RG, int NA, int NBQ, int SRC, bool ONE, bool KEEP>
__global__ __launch_bounds__(512) void k_mx4_mv(const uint8_t *codes, const uint8_t *scales, const uint8_t *x, int S, int NC, uint32_t b_bytes, uint32_t b_col,
                                                uint32_t b_chunk, int n_rg, int rg0, int W, int rounds, Mx4MvRest rest) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int NCP = 16 * NCB, kRed = 8 * RG * NCP * 16;  // columns as computed; floats of one round's slice sums
    constexpr bool kModel = EPI == EPI_QKV || EPI == EPI_RESID || EPI == EPI_SWIGLU, kNorm = EPI == EPI_QKV || EPI == EPI_SWIGLU;
    constexpr bool kTwo = !ONE && kMx4TwoBuffers<NCB, RG>;
    static_assert(SRC == kRegisters ? (4 * NA) % NBQ == 0 : NCB == 1, "a block of the window holds whole turns of B's registers");
    float *red = (float *)smem, *rs = red + (kTwo ? 2 : 1) * kRed, *nscratch = rs + 64;
    unsigned char *lds_b = (unsigned char *)(nscratch + (kNorm ? 1024 : 0));
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const int n = (S + 7) >> 3, s0 = min(wave * n, S), nv = min(n, S - s0), last_rg = n_rg - 1;

    // ---- weights and activations as buffers
    __amdgpu_buffer_rsrc_t cs[RG], ss[RG];
    auto set_slices = [&](int seg) {
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            const size_t at = (size_t)min(rg0 + (seg * W + (int)blockIdx.x) * RG + g, last_rg) * S + s0;
            const int live = ONE || seg < rounds ? nv : 0;
            cs[g] = __builtin_amdgcn_make_buffer_rsrc((void *)(codes + at * 1024), 0, live * 1024, 0x00020000);
            ss[g] = __builtin_amdgcn_make_buffer_rsrc((void *)(scales + at * 64), 0, live * 64, 0x00020000);
        }
    };
    u32x4 A[NA][RG];
    uint32_t E[NA][RG];
    u32x4 B[SRC == kRegisters ? NBQ : 1][NCB];
    auto load_a = [&](int i, u32x4(&c)[RG], uint32_t(&e)[RG]) {
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            c[g] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(cs[g], lane * 16, i * 1024, kNonTemporal));
            e[g] = __builtin_amdgcn_raw_buffer_load_b8(ss[g], lane, i * 64, kNonTemporal);
        }
    };
    // (B is contiguous chunk by chunk: past the slice and past the depth loads read nothing)
    const uint32_t b_from = __builtin_amdgcn_readfirstlane(16 * s0 * b_chunk);
    const uint32_t b_here = __builtin_amdgcn_readfirstlane(min(b_from < b_bytes ? b_bytes - b_from : 0, 16 * nv * b_chunk));
    const __amdgpu_buffer_rsrc_t xs = __builtin_amdgcn_make_buffer_rsrc((void *)(x + b_from), 0, b_here, 0x00020000);
    uint32_t b_at[NCB];
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) b_at[cb] = 16 * cb + col < NC ? (16 * cb + col) * b_col + 4 * kg * b_chunk : kNowhere;
    auto load_b = [&](int i, int t, u32x4(&b)[NCB]) {  // quarter t of super-tile i of the slice
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
            b[cb] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xs, b_at[cb], (16 * i + t) * b_chunk, 0));
    };

    // (what the epilogue needs goes out ahead of the window: loads come back in order)
    const auto &q = late_args<decltype(&k_mx4_mv<EPI, NCB, RG, NA, NBQ, SRC, ONE, KEEP>)>();
    const MvArgs &a = q.a;
    // B to LDS: lines of the slice's bytes, or split rows; l_col and l_chunk: bytes from a column, a chunk to the next there
    const uint32_t line = mx4_lds_line(n, b_chunk);
    const uint32_t l_col = SRC == kLds && b_col != 16 ? line : 16, l_chunk = SRC == kLdsSplit ? 16 * NC : b_chunk;
    unsigned char *lx = lds_b + (size_t)wave * (16 + (SRC == kLds ? (uint32_t)q.lines * line : mx4_lds_line(n, 16 * NC)));
    const uint32_t real = min(b_here, line - 16);  // bytes of a line that exist (kLds)
    if constexpr (SRC == kLds) {
        if (real > 0)
            for (int l = 0; l < q.lines; ++l)
                for (uint32_t p = 0; p < line - 16; p += 1024)  // (a line's last 16 bytes are room between columns, read by nobody)
                    if (p + lane * 16 < line) to_lds<16>(x + (size_t)l * q.line_pitch + b_from + min(p + lane * 16, real - 16), lx + 16 + l * line + p);
    }
    NormPart np;
    NormPart32 np32;
    NormPart64 np64;
    if constexpr (kNorm) {
        if constexpr (NCB <= 3)
            np = mv_norm_load(a);
        else if constexpr (NCB == 8)
            np64 = mv_norm64_load(a);
        else
            np32 = mv_norm32_load(a);
    }
    constexpr int share = 8 / RG;  // wavefronts per row group in a model's epilogue
    constexpr int kPasses = ((NCB <= 3 ? 16 : NCB == 8 ? 64 : 32) / 4 + share - 1) / share;
    constexpr bool kAhead = EPI == EPI_RESID && NCB <= 3;
    const int eg = min(wave / share, RG - 1);
    Residuals<kPasses> X;
    if constexpr (kAhead) X = mv_residuals<kPasses>(a, min(rg0 + (int)blockIdx.x * RG + eg, last_rg), lane, wave - eg * share, share);
    // a call's epilogue: thread tid has four results (J of them to a row and row group)
    constexpr int J = EPI == EPI_GATED ? 2 : 4;
    const int cj = tid % J, cg = tid / J % RG, cr = tid / (J * RG);  // its four, its row group, its row
    u32x4 res = {0u, 0u, 0u, 0u};
    auto request = [&](int seg) {
        const int rg = rg0 + (seg * W + (int)blockIdx.x) * RG + cg, row = 4 * J * rg + 4 * cj;
        if (EPI == EPI_LINEAR && q.out.residual && cr < a.R && rg <= last_rg && row < a.O)
            res = mx4_residual_words(q.out, cr, row, min(a.O - row, 4), mx4_out_by_fours(q.out));
    };
    request(0);
    // rows to split: what most slices hold of the first row is requested ahead of the window and split behind it
    constexpr int kEarly = ONE && NA <= 4 ? 1 : 3;
    float early[SRC == kLdsSplit ? kEarly : 1][8];
    const int mine = 16 * n;
    auto row_chunk = [&](int r, int ch, float *v) {
        mx4_load8<F32T>(q.x32 + r * q.ld_x, 8 * (16 * s0 + ch), ch < mine ? q.K : 0, ((uintptr_t)q.x32 & 15) == 0 && (q.ld_x & 3) == 0, v);
    };
    if constexpr (SRC == kLdsSplit) {
#pragma unroll
        for (int j = 0; j < kEarly; ++j) row_chunk(0, lane + 64 * j, early[j]);
    }
    __builtin_amdgcn_sched_barrier(0);
    set_slices(0);
#pragma unroll
    for (int u = 0; u < NA; ++u) load_a(u, A[u], E[u]);
    if constexpr (SRC == kRegisters) {
#pragma unroll
        for (int u = 0; u < NBQ; ++u) load_b(u >> 2, u & 3, B[u]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (SRC != kRegisters) {
        if (lane == 0) *(u32x4 *)lx = u32x4{0u, 0u, 0u, 0u};
    }
    if constexpr (SRC == kLdsSplit) {
        auto put = [&](int r, int ch, const float *v) {
            if (ch >= mine) return;
            u32x4 t[3];
            mx4_split8(v, t);
#pragma unroll
            for (int j = 0; j < 3; ++j) *(u32x4 *)(lx + 16 + (size_t)(ch * NC + 3 * r + j) * 16) = t[j];
        };
#pragma unroll
        for (int j = 0; j < kEarly; ++j) put(0, lane + 64 * j, early[j]);
        for (int r = 0; r < a.R; ++r)
            for (int ch = lane + (r == 0 ? 64 * kEarly : 0); ch < mine; ch += 64) {
                float v[8];
                row_chunk(r, ch, v);
                put(r, ch, v);
            }
    }
    if constexpr (SRC == kLds) {
        // (the lines have arrived; the window behind them, 2 loads a super-tile and row group, may be on its way)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NA * RG > 63 ? 63 : 2 * NA * RG) : "memory");
        if (real < line - 16)  // zeros past the depth
            for (int l = 0; l < q.lines; ++l)
                for (uint32_t p = real + lane * 16; p < line - 16; p += 1024) *(u32x4 *)(lx + 16 + l * line + p) = u32x4{0u, 0u, 0u, 0u};
    }
    const unsigned char *l_at = col < NC ? lx + 16 + col * l_col + 4 * kg * l_chunk : lx;
    const uint32_t l_step = col < NC ? l_chunk : 0;
    if constexpr (kNorm) {
        if constexpr (NCB <= 3)
            mv_norm_finish(a, np, rs, nscratch);
        else if constexpr (NCB == 8)
            mv_norm64_finish(a, np64, rs, nscratch);
        else
            mv_norm32_finish(a, np32, rs, nscratch);
    }
    const int nb = (n + NA - 1) / NA;
    f32x4 acc[RG][NCB];
    for (int seg = 0; seg < (ONE ? 1 : rounds); ++seg) {
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb) acc[g][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int crg = rg0 + (seg * W + (int)blockIdx.x) * RG + cg, crow = 4 * J * crg + 4 * cj;
        if (seg > 0) request(seg);
        for (int b = 0; b < (ONE ? 1 : nb); ++b) {
            const bool last = b + 1 == nb;
            const int base = b * NA, ahead = last ? 0 : base + NA;  // this block's first super-tile; the next one's
            if (!ONE && last) set_slices(seg + 1);
            each<NA>([&](auto U) {
                constexpr int u = decltype(U)::value;
                // (wavefront-uniform.  With B in registers a window's steps past the slice multiply zeros with zeros: behind a branch the
                // compiler waits for more loads than it has to)
                const bool on = (SRC == kRegisters && !ONE) || base + u < nv;
                each<4>([&](auto T) {
                    constexpr int t = decltype(T)::value, at = 4 * u + t + NBQ;  // at: in quarters from this block's start
                    u32x4(&bb)[NCB] = B[SRC == kRegisters ? (4 * u + t) % NBQ : 0];
                    if (on) {
                        if constexpr (SRC != kRegisters) bb[0] = *(const u32x4 *)(l_at + (16 * (base + u) + t) * l_step);
#pragma unroll
                        for (int g = 0; g < RG; ++g) {
                            const bf16x8 av = mx4_decode(A[u][g][t], __uint_as_float(E[u][g] << 23));
#pragma unroll
                            for (int cb = 0; cb < NCB; ++cb)
                                acc[g][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, bb[cb]), acc[g][cb], 0, 0, 0);
                        }
                    }
                    if constexpr (SRC == kRegisters && !KEEP) {
                        if constexpr (at < 4 * NA)
                            load_b(base + at / 4, at & 3, bb);
                        else if constexpr (!ONE)
                            load_b(ahead + (at - 4 * NA) / 4, at & 3, bb);
                    }
                });
                if constexpr (!ONE) load_a(ahead + u, A[u], E[u]);
            });
        }
        // ---- slice sums to LDS, then all wavefronts share the epilogue
        if (!kTwo && seg > 0) lds_barrier();  // (the previous round's sums are no longer read)
        float *rp = red + (kTwo ? (size_t)(seg & 1) * kRed : 0);
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb) *(f32x4 *)(rp + ((wave * RG + g) * NCP + 16 * cb + col) * 16 + 4 * kg) = acc[g][cb];
        lds_barrier();  // (the next round's loads stay in flight)
        // (every thread adds up four of a column: left to the epilogues, few of whose threads have work, the same additions took 3 us)
        constexpr int slice = RG * NCP * 16;  // floats from one slice to the next
        for (int e = tid; e < RG * NCP * 4; e += 512) {
            f32x4 v = *(const f32x4 *)(rp + 4 * e);
#pragma unroll
            for (int k = 1; k < 8; ++k) v += *(const f32x4 *)(rp + k * slice + 4 * e);
            *(f32x4 *)(rp + 4 * e) = v;
        }
        lds_barrier();
        if constexpr (kModel) {
            const int g = wave / share, rg = rg0 + (seg * W + (int)blockIdx.x) * RG + g;
            if (g < RG && rg <= last_rg) {
                const int NT = q.NT;
                auto y = [&](int r, int j) {
                    const float *w = rp + (g * NCP + NT * r) * 16 + j;
                    return (w[0] + w[16]) + (NT == 3 ? w[32] : 0.f);
                };
                if constexpr (kAhead) {
                    if (seg > 0) X = mv_residuals<kPasses>(a, rg, lane, wave - g * share, share);
                    mv_epilogue<EPI>(a, rg, lane, rs, nullptr, y, wave - g * share, share, X);
                } else {
                    mv_epilogue<EPI>(a, rg, lane, rs, nullptr, y, wave - g * share, share);
                }
            }
        } else {
            const int NT = q.NT;
            auto four = [&](int g, int r, int j) {
                const f32x4 *w = (const f32x4 *)(rp + (g * NCP + NT * r) * 16 + j);
                return NT == 1 ? w[0] : (w[0] + w[4]) + w[8];
            };
            const bool vec = mx4_out_by_fours(q.out);
            // (a thread's first four; more results than threads: many rows of several row groups)
            for (int r = cr; r < a.R; r += 512 / (J * RG) > 0 ? 512 / (J * RG) : 1) {
                if (tid >= 512 / (J * RG) * (J * RG) || crg > last_rg || crow >= a.O) break;
                const int cnt = min(a.O - crow, 4);
                f32x4 v = four(cg, r, 4 * cj);
                if constexpr (EPI == EPI_LINEAR) {
                    if (q.out.residual) {
                        if (r != cr) res = mx4_residual_words(q.out, r, crow, cnt, vec);
                        v += mx4_residual_values(q.out, res, cnt, vec);
                    }
                } else {
                    const f32x4 up = four(cg, r, 8 + 4 * cj);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = mx4_silu(v[k]) * up[k];
                }
                mx4_store4(q.out, r, crow, cnt, vec, v);
            }
        }
    }
}

template <int EPI, int NCB, int RG, int NA, int NBQ, int SRC, bool ONE, bool KEEP = false>
hipError_t launch_mv_t(const Mx4Matrix &w, const Mx4Columns &c, const Mx4MvRest &rest, int rg0, int n_cu, hipStream_t s) {
    constexpr bool kNorm = EPI == EPI_QKV || EPI == EPI_SWIGLU;
    const size_t lds = ((!ONE && kMx4TwoBuffers<NCB, RG> ? 2 : 1) * 8 * RG * 16 * NCB * 16 + 64 + (kNorm ? 1024 : 0)) * 4 +
                       (SRC == kRegisters ? 0 : SRC == kLds ? mx4_lds_bytes(w.K, rest.lines, c.b_chunk) : mx4_lds_bytes(w.K, 1, 16 * c.NC));
    if (lds > 160 * 1024 || ((ONE || KEEP) && (w.S + 7) / 8 > NA)) return hipErrorInvalidValue;
    const auto k = k_mx4_mv<EPI, NCB, RG, NA, NBQ, SRC, ONE, KEEP>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const int units = (rest.a.n_rg - rg0 + RG - 1) / RG, rounds = ONE ? 1 : (units + n_cu - 1) / n_cu, W = (units + rounds - 1) / rounds;
    hipLaunchKernelGGL(k, dim3(W), dim3(512), lds, s, w.codes, w.scales, (const uint8_t *)c.x, w.S, c.NC, c.bytes, c.b_col, c.b_chunk, rest.a.n_rg, rg0, W,
                       rounds, rest);
    return hipGetLastError();
}
// Up to 16 columns, B in LDS.  us, launches back to back, one bf16 row unless said otherwise:
//  * slices of up to 4 super-tiles (depth 4096) or 8: the whole window at once, a row group a workgroup (12288 x 4096 7.2, three to a workgroup 7.6;
//    gate/up of 11008 x 4096 10.8 / 11.4; gate/up of 13824 x 5120 15.0, rounds of two 20.1), unless a workgroup's copy of B outweighs its
//    codes: 9 rows, 12288 x 4096 13.4 / 8.7, gate/up 25.9 / 15.5; 3 fp32 rows, 15360 x 5120 31.0, rounds of two 16.0;
//    with copies of 40 to 56 KB (2 fp32 rows, gate/up; 6 bf16 rows, gate/up) 17.2 / 13.0 and 15.6 / 11.9.
//  * up to 12 (11008), one row group per compute unit: the whole window, 8.0; rounds of windows of 4 9.5.
//  * deeper: rounds of two row groups (8192 x 28672 22.8, 5.5 TB/s).
template <int EPI, int SRC>
hipError_t launch_mv_lds(const Mx4Matrix &w, const Mx4Columns &c, const Mx4MvRest &rest, int rg0, int n_cu, size_t lds_b, hipStream_t s) {
    const int n = (w.S + 7) / 8, n_rg = rest.a.n_rg - rg0;
    const bool light = lds_b <= 40 * 1024 || n_rg <= n_cu;
    if (n <= 4) {
        if (light) return launch_mv_t<EPI, 1, 1, 4, 1, SRC, true>(w, c, rest, rg0, n_cu, s);
        if (n_rg <= 2 * n_cu) return launch_mv_t<EPI, 1, 2, 4, 1, SRC, true>(w, c, rest, rg0, n_cu, s);
        return launch_mv_t<EPI, 1, 3, 4, 1, SRC, true>(w, c, rest, rg0, n_cu, s);
    }
    if (n <= 8 && light) return launch_mv_t<EPI, 1, 1, 8, 1, SRC, true>(w, c, rest, rg0, n_cu, s);
    if (n <= 12 && n_rg <= n_cu) return launch_mv_t<EPI, 1, 1, 12, 1, SRC, true>(w, c, rest, rg0, n_cu, s);
    return launch_mv_t<EPI, 1, 2, 4, 1, SRC, false>(w, c, rest, rg0, n_cu, s);
}

// More columns, or too deep for LDS: B in registers.  us, fp32 rows laid out by a launch of their own (2.2 of it), 9 rows:
//  * two column blocks, slices of up to 4: the whole window with as many row groups as give every compute unit a workgroup (12288 x 4096: three 13.2,
//    one 20.7), beyond that rounds of two that keep B (gate/up 11008: 19.6; whole windows of three 21.7);
//  * deeper: rounds of one row group where that is one round (4096 x 11008: 19.5, of two 24), else of three, else of six (28672 x 8192 gate/up, 32
//    bf16 rows: 72, of three 76).
// The two kernels' times in hundredths of a microsecond a super-tile: this file's, per row group of a compute unit, grows
// with the columns; the other's (swift_mx4_narrow.hip), per round of workgroups of 8 or 16 row groups, much less.  Up to 32 columns and 32
// super-tiles this one streams the weights nearly as fast as memory gives them (70000x4096 4.05 TB/s) and the other is no faster.
bool mx4_narrow_pays(int ncb, int n_rg, int n, int n_cu) {
    if (ncb < 2 || ncb > 6 || (ncb == 2 && n <= 4)) return false;
    const int per = (n_rg + n_cu - 1) / n_cu, rounds = (per + 15) / 16;
    const int few = (ncb == 2 ? 8 : ncb <= 4 ? 16 : 22) * per;
    return few > (ncb == 2 ? 95 : ncb <= 4 ? 119 : per <= 8 ? 103 : 147) * rounds;
}

template <int EPI>
hipError_t launch_mv_e(const Mx4Matrix &w, const Mx4Columns &c, Mx4MvRest rest, int rg0, int n_cu, float *part, hipStream_t s) {
    constexpr bool kModel = EPI == EPI_QKV || EPI == EPI_RESID || EPI == EPI_SWIGLU;
    const int ncb = (c.NC + 15) / 16, n_rg = rest.a.n_rg - rg0, n = (w.S + 7) / 8;
    if (ncb == 1) {
        rest.lines = c.b_col == 16 ? 1 : c.NC;
        const size_t lds_b = mx4_lds_bytes(w.K, rest.lines, c.b_chunk);
        if (lds_b <= kMx4LdsMost) return launch_mv_lds<EPI, kLds>(w, c, rest, rg0, n_cu, lds_b, s);
    }
    const int per = (n_rg + n_cu - 1) / n_cu;  // row groups a compute unit
    if constexpr (EPI == EPI_RESID || EPI == EPI_LINEAR) {
        if (mx4_sliced(c.NC, n_rg, w.S)) return launch_mx4_slices(EPI, w, rest.a, rest.out, c, rest.NT, part, s);
    }
    if constexpr (EPI == EPI_SWIGLU || !kModel) {  // (the other projections of a model do not have that many rows)
        if (c.b_col == 16 && mx4_narrow_pays(ncb, n_rg, n, n_cu)) return launch_mx4_narrow(EPI, w, rest.a, rest.out, c, rest.NT, n_cu, s);
    }
    switch (ncb) {
        case 1:
        case 2:
            if (n <= 4) {
                if (per == 1) return launch_mv_t<EPI, 2, 1, 4, 16, kRegisters, true>(w, c, rest, rg0, n_cu, s);
                if (per == 3) return launch_mv_t<EPI, 2, 3, 4, 16, kRegisters, true>(w, c, rest, rg0, n_cu, s);
                return launch_mv_t<EPI, 2, 2, 4, 16, kRegisters, false, true>(w, c, rest, rg0, n_cu, s);
            }
            if (per == 1) return launch_mv_t<EPI, 2, 1, 4, 8, kRegisters, false>(w, c, rest, rg0, n_cu, s);
            if (per <= 6) return launch_mv_t<EPI, 2, 3, 4, 8, kRegisters, false>(w, c, rest, rg0, n_cu, s);
            return launch_mv_t<EPI, 2, 6, 2, 8, kRegisters, false>(w, c, rest, rg0, n_cu, s);
        case 3:
            if (per == 1) return launch_mv_t<EPI, 3, 1, 2, 8, kRegisters, false>(w, c, rest, rg0, n_cu, s);
            return launch_mv_t<EPI, 3, 2, 4, 8, kRegisters, false>(w, c, rest, rg0, n_cu, s);
        case 4:
            if (per == 1) return launch_mv_t<EPI, 4, 1, 2, 8, kRegisters, false>(w, c, rest, rg0, n_cu, s);
            return launch_mv_t<EPI, 4, 2, 4, 4, kRegisters, false>(w, c, rest, rg0, n_cu, s);
        case 5:
        case 6:
            if (per == 1) return launch_mv_t<EPI, 6, 1, 2, 4, kRegisters, false>(w, c, rest, rg0, n_cu, s);
            return launch_mv_t<EPI, 6, 2, 2, 4, kRegisters, false>(w, c, rest, rg0, n_cu, s);
        case 7:
        case 8:
            if constexpr (kModel) return launch_mv_t<EPI, 8, 1, 2, 4, kRegisters, false>(w, c, rest, rg0, n_cu, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_mx4_mv(int epi, const MvArgs &a, const Mx4Matrix &w, int rg0, int n_cu, float *part, hipStream_t s) {
    const bool bulk = (a.RL & kBulkLayout) != 0;
    const int lrows = layout_rows(a.RL), NT = block_terms(a.RL), NC = NT * lrows, ncb = (NC + 15) / 16;
    if (a.R < 1 || a.R > kMaxBlockRows || (a.rp != 16 && a.rp != 64) || a.R > a.rp || a.R > lrows ||
        (bulk ? (lrows != 32 && lrows != 64) : (lrows != a.R || lrows > kMaxRows)) || (a.rp == 16) != (ncb <= 3) || (a.K & 7) != 0 ||
        w.S != mx4_tiles(a.K) || rg0 < 0 || rg0 >= a.n_rg || a.n_rg > w.n_rg || (epi != EPI_RESID && (!a.pss || a.n_pss < 1)))
        return hipErrorInvalidValue;
    const Mx4Columns c{(const uint16_t *)a.in_s, NC, (uint32_t)(a.K >> 3) * NC * 16, 16, 16u * NC};
    Mx4MvRest rest{};
    rest.a = a;
    rest.NT = NT;
    switch (epi) {
        case EPI_QKV: return launch_mv_e<EPI_QKV>(w, c, rest, rg0, n_cu, part, s);
        case EPI_RESID: return launch_mv_e<EPI_RESID>(w, c, rest, rg0, n_cu, part, s);
        case EPI_SWIGLU: return launch_mv_e<EPI_SWIGLU>(w, c, rest, rg0, n_cu, part, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_mx4_call(int epi, const Mx4CallArgs &c, int n_cu, hipStream_t s) {
    const int NC = c.n * c.terms;
    if (c.n < 1 || NC > kMx4FewColumns) return hipErrorInvalidValue;
    Mx4MvRest rest{};
    rest.a.R = c.n;
    rest.a.O = c.O;
    rest.a.n_rg = c.w.n_rg;
    rest.out = c.out;
    rest.NT = c.terms;
    rest.K = c.w.K;
    const uint32_t pitch = mx4_pitch(NC);
    Mx4Columns cols{c.x, NC, (uint32_t)c.w.S * 16 * pitch * 16, 16, 16 * pitch};
    if (c.direct) {  // the call's own bf16 rows
        cols.bytes = 2u * c.w.K;
        cols.b_col = c.n == 1 ? 16 : 0;  // (lines of their own)
        cols.b_chunk = 16;
        rest.line_pitch = (uint32_t)(2 * c.ld_x);
    }
    if (c.x32) {
        rest.x32 = c.x32;
        rest.ld_x = c.ld_x;
        if (epi == EPI_LINEAR) return launch_mv_lds<EPI_LINEAR, kLdsSplit>(c.w, cols, rest, 0, n_cu, mx4_lds_bytes(c.w.K, 1, 16 * NC), s);
        if (epi == EPI_GATED) return launch_mv_lds<EPI_GATED, kLdsSplit>(c.w, cols, rest, 0, n_cu, mx4_lds_bytes(c.w.K, 1, 16 * NC), s);
        return hipErrorInvalidValue;
    }
    if (epi == EPI_LINEAR) return launch_mv_e<EPI_LINEAR>(c.w, cols, rest, 0, n_cu, c.part, s);
    if (epi == EPI_GATED) return launch_mv_e<EPI_GATED>(c.w, cols, rest, 0, n_cu, c.part, s);
    return hipErrorInvalidValue;
}

}  // namespace swift
