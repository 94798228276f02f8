// Products of 17 to 96 columns with an MXFP4 matrix of many rows, or of a great depth: verification blocks and token trees, batches of rows.
//
// There the kernel of few rows (swift_mx4.hip), which reads B from L2 once for every few row groups, waits for B.  Here a workgroup of 8
// wavefronts, WM x WN of them, shares B through LDS for WM RGW row groups: codes, scales and B of a super-tile (128 k) are one stage
// of a ring of NB, copied straight from memory; a wavefront multiplies RGW row groups with CB column blocks.  An eighth of the
// super-tiles at a time is summed from zero, the eighths then in order, a row's terms after that, as in that kernel: a row comes out
// the same bits from either.
//
// Matrices of few rows and a great depth have an eighth of the super-tiles in each workgroup, and a second launch that adds up
// the eight: a compute unit then reads an eighth of B, where it read all of it.  us, a call of 9 fp32 rows (27 columns) and of 96 bf16 rows,
// with the slices apart and in one workgroup (swift_mx4.hip): 4096 x 11008 17.0 / 20.2 and 24.7 / 34.7, 8192 x 28672 41 / 51; up
// to 64 super-tiles the second launch and the way through memory cost more than that saves (64 rows of 8192 x 8192 27.8 / 24.8, of 4096 x 6144
// 18.8 / 18.1; but 96 rows of 600 x 6144 14.6 / 21.3).  768 row groups: 12288 x 9000, 96 rows 50, one row group more 59.
//
// A turn of the ring costs 0.7 to 1.5 us whatever a workgroup's number (waits and barriers, MFMA and decoding; a deeper ring gains nothing, reading
// the next stage early 3 to 8 %), so it pays only where the workgroups fill the card (mx4_narrow_pays).  Measured against the kernel of
// few rows, us: 32 bf16 rows gate/up of 28672x8192 57.1 / 69.1 (4.4 TB/s), 64 rows 76 / 114, 96 rows of 51200x8192 94 / 157, 96 rows
// gate/up of 11008x4096 33 / 42; but 32 rows there 27 / 18.4.
#include <math.h>

#include "swift_device.h"
#include "swift_mv.h"
#include "swift_mx4.h"
#include "swift_mx4_device.h"

namespace swift {

namespace {

// What is copied in place of chunks past the depth (a code of zero times whatever lies there might be a NaN).
__device__ __align__(16) const unsigned char kZeros[16] = {};

struct Mx4NarrowArgs {
    Mx4Matrix w;
    MvArgs a;
    Mx4Out out;
    int NT, NC;        // terms of a row, columns
    int chunks;        // of eight k that B holds
    uint32_t b_chunk;  // bytes from one to the next
    float *part;       // sums of slices [slice][row group][column][16]
};
constexpr int kSlices = -1;  // an epilogue that writes the sums of a slice of the depth to q.part: k_mx4_join does the rest

constexpr int kVPitch = 20;  // floats of a column's 16 results in LDS
template <int WM_, int RGW_, int CB_, int NB_>
struct Mx4Narrow {
    static constexpr int WM = WM_, RGW = RGW_, CB = CB_, NB = NB_, WN = 8 / WM, TRG = WM * RGW, COLS = WN * CB * 16;
    static constexpr int A_BYTES = TRG * 1024, S_AT = A_BYTES, B_AT = S_AT + 1024, STAGE = B_AT + COLS * 256;
    static constexpr bool PIPE = RGW * CB <= 8;  // the next stage is read into registers while one is multiplied, if there are enough of them
    static constexpr int P = TRG + 1 + COLS / 4, PW = (P + 7) / 8;  // pieces of 1 KB of a stage (the scales' one may be partly empty); of a wavefront
    static constexpr int EPI = WM * COLS * kVPitch * 4, NORM_AT = NB * STAGE > EPI ? NB * STAGE : EPI, BYTES = NORM_AT + (64 + 1024) * 4;
    static_assert(TRG <= 16 && BYTES <= 160 * 1024 && NB >= 3 && (NB - 1) * PW < 64, "ring");
};

// What a product does with the sums of a row group, v [column][kVPitch] in LDS: `waves` wavefronts share it, this is the wave-th.
template <int EPI>
__device__ inline void row_group_results(const Mx4NarrowArgs &q, int rg, const float *v, const float *rs, int lane, int wave, int waves) {
    const MvArgs &a = q.a;
    const int NT = q.NT;
    if constexpr (EPI == EPI_RESID || EPI == EPI_SWIGLU) {
        mv_epilogue<EPI>(a, rg, lane, rs, nullptr, [&](int r, int j) {
            const float *p = v + NT * r * kVPitch + j;
            return (p[0] + p[kVPitch]) + (NT == 3 ? p[2 * kVPitch] : 0.f);
        }, wave, waves);
    } else {
        const bool vec = mx4_out_by_fours(q.out);
        constexpr int J = EPI == EPI_LINEAR ? 4 : 2;  // fours of a row's results
        for (int i = 64 * wave + lane; i < J * a.R; i += 64 * waves) {
            const int r = i / J, j = 4 * (i % J), row = 4 * J * rg + j, cnt = min(max(a.O - row, 0), 4);
            auto sum = [&](int at) {
                const float *p = v + NT * r * kVPitch + at;
                f32x4 y = *(const f32x4 *)p;
                if (NT == 3) y = (y + *(const f32x4 *)(p + kVPitch)) + *(const f32x4 *)(p + 2 * kVPitch);
                return y;
            };
            f32x4 y = sum(j);
            if constexpr (EPI == EPI_LINEAR) {
                if (q.out.residual) y += mx4_residual_values(q.out, mx4_residual_words(q.out, r, row, cnt, vec), cnt, vec);
            } else {
                const f32x4 up = sum(8 + j);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = mx4_silu(y[k]) * up[k];
            }
            mx4_store4(q.out, r, row, cnt, vec, y);
        }
    }
}

template <int EPI, typename L>
__global__ __launch_bounds__(512) void k_mx4_narrow(Mx4NarrowArgs q) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int WM = L::WM, WN = L::WN, RGW = L::RGW, CB = L::CB, NB = L::NB, PW = L::PW, TRG = L::TRG;
    constexpr bool kNorm = EPI == EPI_SWIGLU, kParts = EPI == kSlices;
    const MvArgs &a = q.a;
    float *rs = (float *)(smem + L::NORM_AT), *nscratch = rs + 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WM, wn = wave / WM, col = lane & 15, kg = lane >> 4;
    // slices: workgroup i of every eight has the i-th (they go to the dies in turn, so a die's cache holds the columns of one slice)
    const int S = q.w.S, n = (S + 7) >> 3, s_from = kParts ? min((int)(blockIdx.x & 7) * n, S) : 0, s_to = kParts ? min(s_from + n, S) : S;
    const int rg_tile = (int)(kParts ? blockIdx.x >> 3 : blockIdx.x) * TRG, rg_first = rg_tile + wm * RGW, last_rg = a.n_rg - 1;

    // ---- copies: pieces wave + 8 i (past the last one: that one again, the same bytes), each from a wavefront-uniform base
    const unsigned char *src[PW];
    uint32_t off[PW], step[PW];
    int dst[PW];
    bool is_b[PW];
    int b_ch[PW];  // a piece of B: this lane's chunk of the super-tile
#pragma unroll
    for (int i = 0; i < PW; ++i) {
        const int p = min(wave + 8 * i, L::P - 1);
        is_b[i] = p > TRG;
        b_ch[i] = 0;
        dst[i] = p < TRG ? p * 1024 : p == TRG ? L::S_AT : L::B_AT + (p - TRG - 1) * 1024;
        if (p < TRG) {
            src[i] = q.w.codes + (size_t)min(rg_tile + p, last_rg) * S * 1024;
            off[i] = lane * 16;
            step[i] = 1024;
        } else if (p == TRG) {
            src[i] = q.w.scales + (size_t)rg_tile * S * 64;
            off[i] = (uint32_t)(min(rg_tile + min(lane >> 2, TRG - 1), last_rg) - rg_tile) * S * 64 + (lane & 3) * 16;
            step[i] = 64;
        } else {
            const int unit = (p - TRG - 1) * 64 + lane, ch = unit / L::COLS, c = min(unit - ch * L::COLS, q.NC - 1);  // LDS: [quarter][kg][column]
            b_ch[i] = 4 * (ch & 3) + (ch >> 2);
            src[i] = (const unsigned char *)(const uint16_t *)a.in_s;
            off[i] = b_ch[i] * q.b_chunk + c * 16;
            step[i] = 16 * q.b_chunk;
        }
        off[i] += s_from * step[i];
    }
    const bool ragged = q.chunks < 16 * S;
    auto issue = [&](int s, int slot) {
        if (ragged && s == S - 1) {
#pragma unroll
            for (int i = 0; i < PW; ++i)
                to_lds<16>(is_b[i] && 16 * s + b_ch[i] >= q.chunks ? kZeros : src[i] + (size_t)off[i], smem + slot + dst[i]);
        } else {
#pragma unroll
            for (int i = 0; i < PW; ++i) to_lds<16>(src[i] + (size_t)off[i], smem + slot + dst[i]);
        }
        if (s + 1 < s_to) {  // (past the last super-tile: that one again, which nobody reads)
#pragma unroll
            for (int i = 0; i < PW; ++i) off[i] += step[i];
        }
    };
    auto lds_sync = [&]() {
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wavefront's LDS reads are done
        asm volatile("s_barrier" ::: "memory");
    };
    if constexpr (kNorm) {
        if (a.rp == 16)
            mv_norm_finish(a, mv_norm_load(a), rs, nscratch);
        else
            mv_norm32_finish(a, mv_norm32_load(a), rs, nscratch);
        __builtin_amdgcn_sched_barrier(0);
    }
    f32x4 acc[RGW][CB], done[RGW][CB];
#pragma unroll
    for (int g = 0; g < RGW; ++g)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[g][c] = done[g][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    const unsigned char *a_at = smem + wm * RGW * 1024 + lane * 16, *s_at = smem + L::S_AT + wm * RGW * 64 + lane;
    const unsigned char *b_at = smem + L::B_AT + (kg * L::COLS + wn * CB * 16 + col) * 16;
    struct Stage {
        u32x4 code[RGW];
        uint32_t e[RGW];
        bf16x8 b[4][CB];
    };
    auto read = [&](Stage &f, int at) {
#pragma unroll
        for (int g = 0; g < RGW; ++g) {
            f.code[g] = *(const u32x4 *)(a_at + at + g * 1024);
            f.e[g] = *(s_at + at + g * 64);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < CB; ++c) f.b[t][c] = *(const bf16x8 *)(b_at + at + t * L::COLS * 64 + c * 256);
    };
    int cur = 0, left = n;
    auto multiply = [&](int s, const Stage &f) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int g = 0; g < RGW; ++g) {
                const bf16x8 av = mx4_decode(f.code[g][t], __uint_as_float(f.e[g] << 23));
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[g][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, f.b[t][c], acc[g][c], 0, 0, 0);
            }
        if (--left == 0 || s + 1 == s_to) {  // a slice's end
            left = n;
#pragma unroll
            for (int g = 0; g < RGW; ++g)
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    done[g][c] += acc[g][c];
                    acc[g][c] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
        }
    };
    auto turn = [&](int s, const Stage &f, Stage &next) {
        // The next stage has landed for everybody, and everybody has this one in registers: its slot takes the one NB further on.
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * PW) : "memory");
        lds_sync();
        __builtin_amdgcn_sched_barrier(0);
        issue(min(s + NB, s_to - 1), cur);
        cur = cur + L::STAGE == NB * L::STAGE ? 0 : cur + L::STAGE;
        read(next, cur);
        multiply(s, f);
    };
    if (s_from < s_to) {  // (a short depth has empty slices: zeros)
        for (int i = 0; i < (L::PIPE ? NB : NB - 1); ++i) issue(min(s_from + i, s_to - 1), i * L::STAGE);
        if constexpr (L::PIPE) {
            Stage even, odd;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 1) * PW) : "memory");
            lds_sync();
            read(even, 0);
            for (int s = s_from; s < s_to; s += 2) {
                turn(s, even, odd);
                if (s + 1 < s_to) turn(s + 1, odd, even);
            }
        } else {
            int prev = (NB - 1) * L::STAGE;
            Stage f;
            for (int s = s_from; s < s_to; ++s) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * PW) : "memory");
                lds_sync();
                __builtin_amdgcn_sched_barrier(0);
                issue(min(s + NB - 1, s_to - 1), prev);
                read(f, cur);
                multiply(s, f);
                prev = cur;
                cur = cur + L::STAGE == NB * L::STAGE ? 0 : cur + L::STAGE;
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (stages that were asked for past the last)
    }
    if constexpr (kParts) {
#pragma unroll
        for (int g = 0; g < RGW; ++g)
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const int at = wn * CB * 16 + 16 * c + col;
                if (rg_first + g <= last_rg && at < q.NC)
                    *(f32x4 *)(q.part + (((size_t)(blockIdx.x & 7) * a.n_rg + rg_first + g) * q.NC + at) * 16 + 4 * kg) = done[g][c];
            }
    } else {
        // a row group of every wavefront row at a time through LDS, [wavefront row][column][16]
        __syncthreads();
        float *v = (float *)smem + (size_t)wm * L::COLS * kVPitch;
#pragma unroll
        for (int g = 0; g < RGW; ++g) {
            if (g > 0) __syncthreads();
#pragma unroll
            for (int c = 0; c < CB; ++c) *(f32x4 *)(v + (wn * CB * 16 + 16 * c + col) * kVPitch + 4 * kg) = done[g][c];
            __syncthreads();
            if (rg_first + g <= last_rg) row_group_results<EPI>(q, rg_first + g, v, rs, lane, wn, WN);
        }
    }
}

// The slices' sums of a row group, and what a product does with them.
template <int EPI>
__global__ __launch_bounds__(512) void k_mx4_join(Mx4NarrowArgs q) {
    __shared__ __align__(16) float v[kMx4FewColumns * kVPitch];
    const MvArgs &a = q.a;
    const int tid = threadIdx.x, groups = a.n_rg, four = tid & 3, col = tid >> 2;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (col < q.NC) {
        const float *p = q.part + ((size_t)blockIdx.x * q.NC + col) * 16 + 4 * four;
        f32x4 part[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) part[i] = *(const f32x4 *)(p + (size_t)i * groups * q.NC * 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) y += part[i];
    }
    if (col < q.NC) *(f32x4 *)(v + col * kVPitch + 4 * four) = y;
    __syncthreads();
    row_group_results<EPI>(q, (int)blockIdx.x, v, nullptr, tid & 63, tid >> 6, 8);
}

template <int EPI, typename L>
hipError_t launch_tile(const Mx4NarrowArgs &q, hipStream_t s) {
    const int tiles = (q.a.n_rg + L::TRG - 1) / L::TRG * (EPI == kSlices ? 8 : 1);
    const hipError_t e = hipFuncSetAttribute((const void *)k_mx4_narrow<EPI, L>, hipFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mx4_narrow<EPI, L>), dim3(tiles), dim3(512), L::BYTES, s, q);
    return hipGetLastError();
}

template <int EPI>
hipError_t launch_columns(const Mx4NarrowArgs &q, int n_cu, hipStream_t s) {
    if (q.NC <= 32) return launch_tile<EPI, Mx4Narrow<8, 2, 2, 5>>(q, s);
    if (q.NC <= 64) return launch_tile<EPI, Mx4Narrow<4, 4, 2, 4>>(q, s);
    if (q.a.n_rg <= 8 * n_cu) return launch_tile<EPI, Mx4Narrow<4, 2, 3, 4>>(q, s);
    return launch_tile<EPI, Mx4Narrow<4, 4, 3, 3>>(q, s);
}

template <int EPI>
hipError_t launch_slices(const Mx4NarrowArgs &q, hipStream_t s) {
    const hipError_t e = q.NC <= 32   ? launch_tile<kSlices, Mx4Narrow<8, 1, 2, 4>>(q, s)
                         : q.NC <= 64 ? launch_tile<kSlices, Mx4Narrow<4, 2, 2, 4>>(q, s)
                                      : launch_tile<kSlices, Mx4Narrow<4, 2, 3, 4>>(q, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mx4_join<EPI>), dim3(q.a.n_rg), dim3(512), 0, s, q);
    return hipGetLastError();
}

Mx4NarrowArgs narrow_args(const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, const Mx4Columns &c, int NT) {
    Mx4NarrowArgs q{};
    q.w = w;
    q.a = a;
    q.a.in_s = (const uint16_t *)c.x;
    q.out = out;
    q.NT = NT;
    q.NC = c.NC;
    q.chunks = (int)(c.bytes / c.b_chunk);
    q.b_chunk = c.b_chunk;
    return q;
}

}  // namespace

hipError_t launch_mx4_narrow(int epi, const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, const Mx4Columns &c, int NT, int n_cu, hipStream_t s) {
    if (c.NC < 1 || c.NC > kMx4FewColumns || c.b_col != 16) return hipErrorInvalidValue;
    const Mx4NarrowArgs q = narrow_args(w, a, out, c, NT);
    switch (epi) {
        case EPI_SWIGLU: return launch_columns<EPI_SWIGLU>(q, n_cu, s);
        case EPI_LINEAR: return launch_columns<EPI_LINEAR>(q, n_cu, s);
        case EPI_GATED: return launch_columns<EPI_GATED>(q, n_cu, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_mx4_slices(int epi, const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, const Mx4Columns &c, int NT, float *part, hipStream_t s) {
    if (c.NC < 1 || c.NC > kMx4FewColumns || c.b_col != 16 || !part) return hipErrorInvalidValue;
    Mx4NarrowArgs q = narrow_args(w, a, out, c, NT);
    q.part = part;
    switch (epi) {
        case EPI_RESID: return launch_slices<EPI_RESID>(q, s);
        case EPI_LINEAR: return launch_slices<EPI_LINEAR>(q, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace swift
