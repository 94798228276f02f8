// Products of many rows with an MXFP4 matrix: a blocked matrix product on the matrix cores, for prompt macro blocks of a model and for calls.
//
// The rows come in sub-blocks of 128 columns (64 rows of two bf16 terms in a model's prompt; 128 bf16 rows or 42 fp32 rows of three terms in a
// call), laid out as the B operand.  A workgroup of 8 wavefronts, WM x WN, owns WM RGW 16-row groups of weights times WN CB 16 columns (one or two
// sub-blocks); a wavefront RGW row groups times CB column blocks, RGW CB accumulator tiles.  Codes are decoded to bf16 in
// registers, so a tile is kept wide enough that a decoded operand meets several column blocks, and high enough that LDS, which moves 128
// bytes a clock, is not asked for more than half of that.  Both operands come straight from memory into LDS rings: B in stages of Q
// times 32 k (quarter t of a super-tile: the t-th quarter of every lane's block, see swift_mx4.h), codes and scales in
// super-tiles of 128 k, two deep.  One barrier a stage, with what is multiplied first behind it in registers already: a barrier costs
// 0.15 us whatever lies between two of them, so small tiles have longer stages.  Within a stage the next column blocks' operands are
// read while the last ones' are multiplied, and the next quarter's codes are decoded between the matrix instructions.
#include "swift_gemm.h"
#include "swift_mx4.h"
#include "swift_mx4_device.h"

namespace swift {

namespace {

struct Mx4GemmArgs {
    Mx4Matrix w;
    MvArgs a;
    MacroArgs ma;
    Mx4Out out;
    int rg0;        // first row group
    int MT, NN;     // row tiles, column tiles
    int terms;      // of a call's rows
};

constexpr int kVPitch = 20;  // floats of a column's 16 results in LDS
template <int WM_, int RGW_, int CB_, int Q_, int NB_>
struct Mx4Tile {
    static constexpr int WM = WM_, RGW = RGW_, CB = CB_, Q = Q_, NB = NB_;  // NB: stages of B's ring
    static constexpr int WN = 8 / WM, SUBS = WN * CB / 8, TRG = WM * RGW;
    static constexpr int HB = CB < 4 ? CB : 4, PARTS = CB / HB;  // column blocks read at a time, such parts of a quarter
    static constexpr int PER = 4 / Q;                            // stages of a super-tile
    static constexpr int B_STAGE = SUBS * Q * 8192, A_SLOT = TRG * 1024, SP = (RGW + 3) / 4, S_SLOT = WM * SP * 256;  // SP: copies of a wavefront's scales, four row groups each
    static constexpr int A_AT = NB * B_STAGE, S_AT = A_AT + 2 * A_SLOT, RING = S_AT + 2 * S_SLOT;
    static constexpr int EPI = WM * SUBS * 128 * kVPitch * 4;  // the epilogue of calls: a row group's results per wavefront row
    static constexpr int NORM_AT = RING > EPI ? RING : EPI;
    static constexpr int BYTES = NORM_AT + (128 + kNormFloats) * 4;
    static constexpr int AC = (RGW + WN - 1) / WN;     // row groups' codes that a wavefront copies
    static constexpr int AP = AC + SP, PB = SUBS * Q;   // its copies per super-tile of weights, per stage of B
    static_assert(BYTES <= 160 * 1024, "LDS");
    static_assert(SUBS == 1 || SUBS == 2, "columns");
    // The codes of the super-tile after the next are asked for in a super-tile's first stage, ahead of a stage of B that has landed by the time
    // they are read, with the third quarter of the next super-tile (whose stage waits for the B behind it).
    static_assert(NB >= 3 && NB <= (PER == 4 ? 8 : 2 * PER + 1), "ring");
    // A wavefront's copies issued after those of stage i + 1, when stage i begins: those of the NB - 3 stages before i.  ph: i modulo PER.
    static constexpr int ahead(int ph) {
        int n = 0;
        for (int j = 1; j <= NB - 3; ++j) n += PB + ((ph - j + 4 * PER) % PER == 0 ? AP : 0);
        return n;
    }
    // The same in the last two super-tiles, whose 2 PER stages are numbered u: copies end with the last stage.
    static constexpr int tail_ahead(int u) {
        int n = 0;
        for (int j = 1; j <= NB - 3; ++j) {
            const int at = u - j;  // issued then: stage at + NB - 1
            n += (at + NB - 1 < 2 * PER ? PB : 0) + (at < 0 && (at + 4 * PER) % PER == 0 ? AP : 0);
        }
        return n;
    }
};

template <int EPI, typename L>
__global__ __launch_bounds__(512) void k_mx4_gemm(Mx4GemmArgs q) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int WM = L::WM, WN = L::WN, RGW = L::RGW, CB = L::CB, Q = L::Q, HB = L::HB, PARTS = L::PARTS, PER = L::PER, NB = L::NB, AC = L::AC;
    constexpr bool kModel = EPI == EPI_QKV || EPI == EPI_RESID || EPI == EPI_SWIGLU, kNorm = EPI == EPI_QKV || EPI == EPI_SWIGLU;
    const MvArgs &a = q.a;
    const MacroArgs &ma = q.ma;
    float *rs = (float *)(smem + L::NORM_AT), *nscratch = rs + 128;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WM, wn = wave / WM, col = lane & 15, kg = lane >> 4;
    const int ws = wn * CB / 8, c0 = wn * CB % 8;  // its sub-block of the tile, its first column block there
    // the column tiles of a row tile sit next to each other on one die (workgroup ids go round the eight dies): they share its weights
    const int id = blockIdx.x, qd = id >> 3, nt = qd % q.NN, mt = (qd / q.NN) * 8 + (id & 7);
    if (mt >= q.MT) return;
    const int S = q.w.S, tiles = max(S, 2), rg_first = q.rg0 + (mt * WM + wm) * RGW, last_rg = a.n_rg - 1;
    const int sub0 = L::SUBS * nt, sub = min(sub0 + ws, ma.S - 1);

    // ---- copies: wavefront-uniform bases, and a lane's offset from them in the next piece to be asked for
    const unsigned char *a_src[AC], *b_src[L::SUBS];
    int a_dst[AC];
#pragma unroll
    for (int i = 0; i < AC; ++i) {
        const int g = min(i * WN + wn, RGW - 1);  // (RGW no multiple of WN: one is copied twice, the same bytes)
        a_src[i] = q.w.codes + (size_t)min(rg_first + g, last_rg) * S * 1024;
        a_dst[i] = L::A_AT + (wm * RGW + g) * 1024;
    }
    const unsigned char *s_src = q.w.scales + (size_t)min(rg_first, last_rg) * S * 64;
    uint32_t s_off[L::SP];
#pragma unroll
    for (int i = 0; i < L::SP; ++i)
        s_off[i] = (uint32_t)(min(rg_first + min(4 * i + (lane >> 4), RGW - 1), last_rg) - min(rg_first, last_rg)) * S * 64 + 4 * (lane & 15);
    const int bg = wave >> 1, bh = wave & 1;  // chunk group and half of the columns that it copies
#pragma unroll
    for (int i = 0; i < L::SUBS; ++i)
        b_src[i] = (const unsigned char *)(a.in_s + (size_t)min(sub0 + i, ma.S - 1) * ma.in_s) + bg * 8192 + bh * 1024;
    uint32_t b_off = lane * 16, a_off = 0;
    auto issue_a = [&](int s) {  // (past the last super-tile: that one again)
        const int slot = s & 1;
#pragma unroll
        for (int i = 0; i < AC; ++i) to_lds<16>(a_src[i] + (size_t)(a_off + lane * 16), smem + a_dst[i] + slot * L::A_SLOT);
#pragma unroll
        for (int i = 0; i < L::SP; ++i)
            to_lds<4>(s_src + (size_t)((a_off >> 4) + s_off[i]), smem + L::S_AT + slot * L::S_SLOT + (wm * L::SP + i) * 256);  // (the same bytes from each of the WN wavefronts)
        if (s + 1 < S) a_off += 1024;
    };
    auto issue_b = [&](auto PH, int slot) {  // PH: the stage's number in its super-tile
#pragma unroll
        for (int u = 0; u < Q; ++u)
#pragma unroll
            for (int i = 0; i < L::SUBS; ++i)
                to_lds<16>(b_src[i] + (size_t)(b_off + u * 2048), smem + slot + (u * L::SUBS + i) * 8192 + wave * 1024);
        b_off += Q * 2048 + (decltype(PH)::value == PER - 1 ? 12 * 2048 : 0);
    };
    auto lds_sync = [&]() {
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wavefront's LDS reads are done
        asm volatile("s_barrier" ::: "memory");
    };

    // ---- operands
    const unsigned char *b_base = smem + ws * 8192 + kg * 2048 + (16 * c0 + col) * 16;
    const unsigned char *a_base = smem + L::A_AT + wm * RGW * 1024 + lane * 16;
    const unsigned char *s_base = smem + L::S_AT + wm * L::SP * 256 + lane;
    f32x4 acc[RGW][CB];
    u32x4 code[RGW], code_n[RGW], b[2][HB];
    uint32_t sc[RGW], sc_n[RGW];
    bf16x8 av[2][RGW];  // by the parity of the quarter
    auto read_b = [&](u32x4(&d)[HB], int slot, int u, int part) {  // part of the u-th quarter of a stage
#pragma unroll
        for (int c = 0; c < HB; ++c) d[c] = *(const u32x4 *)(b_base + slot + u * L::SUBS * 8192 + (HB * part + c) * 256);
    };
    auto read_a = [&](int s, u32x4(&c)[RGW], uint32_t(&e)[RGW]) {
#pragma unroll
        for (int g = 0; g < RGW; ++g) {
            c[g] = *(const u32x4 *)(a_base + (s & 1) * L::A_SLOT + g * 1024);
            e[g] = *(s_base + (s & 1) * L::S_SLOT + g * 64);
        }
    };

    int prev = (NB - 1) * L::B_STAGE, cur = 0, next = L::B_STAGE;
    // One stage, number PH of super-tile s.  Waits until the next one has landed (ALLOW: this wavefront's copies that may still be on their
    // way), for everybody.
    auto stage = [&](auto PH, auto ISSUE_A, auto ISSUE_B, auto ALLOW, int s) {
        constexpr int ph = decltype(PH)::value;
        constexpr bool ia = decltype(ISSUE_A)::value, ib = decltype(ISSUE_B)::value;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(ALLOW)::value) : "memory");
        lds_sync();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (ia) issue_a(s + 2);
        if constexpr (ib) issue_b(std::integral_constant<int, (ph + NB - 1) % PER>(), prev);  // stage NB - 1 further on
        each<Q * PARTS>([&](auto I) {
            constexpr int i = decltype(I)::value, u = i / PARTS, h = i % PARTS, t = ph * Q + u, p = t & 1, n = i + 1;
            // the next operands: of this stage, or the first of the next one
            if constexpr (n < Q * PARTS)
                read_b(b[n & 1], cur, n / PARTS, n % PARTS);
            else
                read_b(b[n & 1], next, 0, 0);
            if constexpr (t == 2 && h == 0) read_a(s + 1, code_n, sc_n);
#pragma unroll
            for (int g = 0; g < RGW; ++g) {
                if constexpr (h == PARTS - 1)
                    av[p ^ 1][g] = mx4_decode(t == 3 ? code_n[g][0] : code[g][(t + 1) & 3], __uint_as_float((t == 3 ? sc_n[g] : sc[g]) << 23));
#pragma unroll
                for (int c = 0; c < HB; ++c)
                    acc[g][HB * h + c] =
                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[p][g], __builtin_bit_cast(bf16x8, b[i & 1][c]), acc[g][HB * h + c], 0, 0, 0);
            }
            // two matrix instructions, the copies; then a read and some of the decoding behind each matrix instruction
            if constexpr (i == 0 && (ia || ib)) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x020, (ib ? L::PB : 0) + (ia ? L::AP : 0), 0);
            }
#pragma unroll
            for (int j = 0; j < HB * RGW; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, CB == 2 ? 4 : 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        static_assert(Q * PARTS == 2 || Q * PARTS == 4, "the two sets of operands change places within a stage");
        if constexpr (ph == PER - 1) {
#pragma unroll
            for (int g = 0; g < RGW; ++g) {
                code[g] = code_n[g];
                sc[g] = sc_n[g];
            }
        }
        prev = cur;
        cur = next;
        next = next + L::B_STAGE == NB * L::B_STAGE ? 0 : next + L::B_STAGE;
    };

    if constexpr (kNorm) {
        const GemmNorm np = gemm_norm_load(a, ma, sub0);
        gemm_norm_scales(a, gemm_norm_sum(a, ma, sub0, np), rs, nscratch);
        __builtin_amdgcn_sched_barrier(0);
    }
    issue_a(0);
    issue_a(1);
    each<NB - 1>([&](auto I) { issue_b(std::integral_constant<int, decltype(I)::value % PER>(), decltype(I)::value * L::B_STAGE); });
#pragma unroll
    for (int g = 0; g < RGW; ++g)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[g][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 3) * L::PB) : "memory");  // stages 0 and 1
    lds_sync();
    read_a(0, code, sc);
    read_b(b[0], 0, 0, 0);
#pragma unroll
    for (int g = 0; g < RGW; ++g) av[0][g] = mx4_decode(code[g][0], __uint_as_float(sc[g] << 23));
    int s = 0;
    for (; s + 2 < tiles; ++s)
        each<PER>([&](auto I) {
            constexpr int ph = decltype(I)::value;
            stage(I, std::bool_constant<ph == 0>(), std::true_type(), std::integral_constant<int, L::ahead(ph)>(), s);
        });
    // the last two super-tiles (the last stage reads operands that nobody needs)
    each<2 * PER>([&](auto I) {
        constexpr int u = decltype(I)::value;
        stage(std::integral_constant<int, u % PER>(), std::false_type(), std::bool_constant<(u + NB - 1 < 2 * PER)>(),
              std::integral_constant<int, L::tail_ahead(u)>(), s + u / PER);
    });

    // ---- epilogue
    __syncthreads();  // the rings are no longer read
    const bool live = sub0 + ws < ma.S;
    const int rows = sub == ma.S - 1 ? ma.rows_last : kModel ? 64 : 128 / q.terms;
    if constexpr (kModel) {
        if (!live) return;
        MvArgs as = a;
        as.R = rows;
        as.pos0 = a.pos0 + 64 * sub;
        if (a.out_f32) as.out_f32 = a.out_f32 + (size_t)sub * ma.out_f32;
        if (a.out_s) as.out_s = a.out_s + (size_t)sub * ma.out_s;
        if (a.pss_out) as.pss_out = a.pss_out + (size_t)sub * ma.pss_out;
        each<CB / 4>([&](auto H) {
            constexpr int h = decltype(H)::value;
            const int r0 = 8 * c0 + 32 * h;  // 64 columns: 32 rows
            if (r0 >= rows) return;
            auto y = [&](int g, f32x4(&v)[2]) {
                const f32x4 z[4] = {acc[g][4 * h], acc[g][4 * h + 1], acc[g][4 * h + 2], acc[g][4 * h + 3]};
                fold_terms(z, col, v);
            };
            if constexpr (EPI == EPI_RESID) {
                gemm_resid<RGW>(as, rg_first, r0, lane, y);
            } else {
                float scale[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) scale[c] = rs[64 * ws + r0 + gemm_row(c, col)];
                if constexpr (EPI == EPI_QKV) {
                    gemm_qkv<RGW>(as, rg_first, r0, lane, scale, (uint16_t *)smem + (size_t)wave * 1024, y);
                } else {
#pragma unroll
                    for (int g = 0; g < RGW; ++g) {
                        if (rg_first + g >= a.n_rg) break;
                        f32x4 v[2];
                        y(g, v);
                        gemm_swiglu(as, rg_first + g, r0, lane, scale, v);
                    }
                }
            }
        });
    } else {
        const int r0 = sub * (128 / q.terms);
        const Mx4Out o = mx4_out_from(q.out, r0);
        const bool vec = mx4_out_by_fours(o);
        if (q.terms == 1) {
            // a column is a row of the result, and a lane holds four of its values in a row (gate and up: after an exchange of lanes)
            if (!live) return;
            constexpr int N = EPI == EPI_LINEAR ? CB : CB / 2;  // results of four of a lane for a row group
            auto place = [&](int g, int c, int &r, int &row) {
                if (EPI == EPI_LINEAR) {
                    r = 16 * (c0 + c) + col;
                    row = 16 * (rg_first + g) + 4 * kg;
                } else {
                    r = 16 * (c0 + 2 * c + (kg >> 1)) + col;
                    row = 8 * (rg_first + g) + 4 * (kg & 1);
                }
                return r < rows ? min(max(a.O - row, 0), 4) : 0;
            };
            u32x4 res[2][N];  // a row group's residual values, requested while the one before it is written
            auto request = [&](int g) {
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    int r, row;
                    const int n = place(g, c, r, row);
                    res[g & 1][c] = mx4_residual_words(o, r, row, n, vec);
                }
            };
            if (EPI == EPI_LINEAR && o.residual) request(0);
#pragma unroll
            for (int g = 0; g < RGW; ++g) {
                if (EPI == EPI_LINEAR && o.residual && g + 1 < RGW) request(g + 1);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    int r, row;
                    const int n = place(g, c, r, row);
                    f32x4 v;
                    if constexpr (EPI == EPI_LINEAR) {
                        v = acc[g][c];
                        if (o.residual) v += mx4_residual_values(o, res[g & 1][c], n, vec);
                    } else {
                        f32x4 ga = acc[g][2 * c], up = acc[g][2 * c + 1];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float x = ga[i], y = up[i];
                            swap32(x, y);  // kg < 2: gate and up of column block 2 c; else of 2 c + 1
                            v[i] = mx4_silu(x) * y;
                        }
                    }
                    mx4_store4(o, r, row, n, vec, v);
                }
            }
        } else {
            // a row group's results through LDS, [wavefront row][sub-block][column][16], then a row's terms are added in order by the
            // wavefronts that share the sub-block
            constexpr int SHARE = 8 / CB, J = EPI == EPI_LINEAR ? 4 : 2;  // fours of a row's results
            float *v = (float *)smem + (size_t)(wm * L::SUBS + ws) * 128 * kVPitch;
#pragma unroll
            for (int g = 0; g < RGW; ++g) {
                if (g > 0) __syncthreads();
#pragma unroll
                for (int c = 0; c < CB; ++c) *(f32x4 *)(v + (16 * (c0 + c) + col) * kVPitch + 4 * kg) = acc[g][c];
                __syncthreads();
                if (!live) continue;
                for (int i = 64 * (wn % SHARE) + lane; i < J * rows; i += 64 * SHARE) {
                    const int r = i / J, j = 4 * (i % J), row = 4 * J * (rg_first + g) + j, n = min(max(a.O - row, 0), 4);
                    auto sum = [&](int at) {
                        const float *p = v + 3 * r * kVPitch + at;
                        return (*(const f32x4 *)p + *(const f32x4 *)(p + kVPitch)) + *(const f32x4 *)(p + 2 * kVPitch);
                    };
                    f32x4 y = sum(j);
                    if constexpr (EPI == EPI_LINEAR) {
                        if (o.residual) y += mx4_residual_values(o, mx4_residual_words(o, r, row, n, vec), n, vec);
                    } else {
                        const f32x4 up = sum(8 + j);
#pragma unroll
                        for (int k = 0; k < 4; ++k) y[k] = mx4_silu(y[k]) * up[k];
                    }
                    mx4_store4(o, r, row, n, vec, y);
                }
            }
        }
    }
}

template <int EPI, typename L>
hipError_t launch_tile(Mx4GemmArgs q, hipStream_t s) {
    q.MT = (q.a.n_rg - q.rg0 + L::TRG - 1) / L::TRG;
    q.NN = (q.ma.S + L::SUBS - 1) / L::SUBS;
    const hipError_t e = hipFuncSetAttribute((const void *)k_mx4_gemm<EPI, L>, hipFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mx4_gemm<EPI, L>), dim3((unsigned)((q.MT + 7) / 8 * 8 * q.NN)), dim3(512), L::BYTES, s, q);
    return hipGetLastError();
}

// The tiles, rows x columns, and what they cost: us per super-tile (from the differences of depths of 4096, 8192 and 16384) and per workgroup
// beside them (start, first stages, epilogue).  The matrix instructions alone take 1.86, 0.93, 0.70 and 0.47: the smaller tiles read more
// of LDS for each of them.  1024 x 5120 x 5120, bf16, us with each: 112, 69, 63, 97; 512 x 4096 x 4096: 83, 48, 42, 38; 2048 x 8192 x 8192: 189
// (1456 TFLOP/s), 207, 228, 283.
using Tile256x256 = Mx4Tile<4, 4, 8, 1, 7>;
using Tile256x128 = Mx4Tile<4, 4, 4, 2, 5>;
using Tile192x128 = Mx4Tile<4, 3, 4, 2, 5>;
using Tile128x128 = Mx4Tile<2, 4, 2, 4, 3>;
struct TileCost {
    int rows, cols;
    double tile, fixed;
};
constexpr TileCost kTiles[] = {{256, 256, 1.95, 13.0}, {256, 128, 1.06, 9.0}, {192, 128, 0.86, 8.5}, {128, 128, 0.90, 5.0}};

// The cheapest in rounds of one workgroup per compute unit.  tiles: those a launch can take (the narrowest is a call's only).
int choose(const Mx4GemmArgs &q, int n_cu, int tiles) {
    int best = 0;
    double least = 1e30;
    for (int i = 0; i < tiles; ++i) {
        const TileCost &t = kTiles[i];
        const int64_t groups = (int64_t)((16 * (q.a.n_rg - q.rg0) + t.rows - 1) / t.rows) * ((128 * q.ma.S + t.cols - 1) / t.cols);
        const double us = (double)((groups + n_cu - 1) / n_cu) * (q.w.S * t.tile + t.fixed);
        if (us < least) {
            least = us;
            best = i;
        }
    }
    return best;
}

template <int EPI>
hipError_t launch_chosen(const Mx4GemmArgs &q, int n_cu, hipStream_t s) {
    constexpr bool kCall = EPI == EPI_LINEAR || EPI == EPI_GATED;
    const int c = choose(q, n_cu, kCall ? 4 : 3);
    if constexpr (kCall)
        if (c == 3) return launch_tile<EPI, Tile128x128>(q, s);
    if (c == 2) return launch_tile<EPI, Tile192x128>(q, s);
    return c == 0 ? launch_tile<EPI, Tile256x256>(q, s) : launch_tile<EPI, Tile256x128>(q, s);
}

}  // namespace

hipError_t launch_mx4_macro(int epi, const MvArgs &a, const MacroArgs &ma, const Mx4Matrix &w, int rg0, int n_cu, hipStream_t s) {
    if (ma.S < 1 || ma.S > kMacroSub || ma.rows_last < 1 || ma.rows_last > 64 || a.RL != (64 | kBulkLayout) || a.rp != 64 || a.tree || a.q_s ||
        a.head0 != 0 || (a.K & 7) != 0 || w.S != mx4_tiles(a.K) || rg0 < 0 || rg0 >= a.n_rg || a.n_rg > w.n_rg ||
        (epi == EPI_RESID ? !a.gain_next || !a.pss_out || (a.O & 7) != 0 : !a.pss || a.n_pss < 1))
        return hipErrorInvalidValue;
    Mx4GemmArgs q{};
    q.w = w;
    q.a = a;
    q.ma = ma;
    q.rg0 = rg0;
    q.terms = 2;
    switch (epi) {
        case EPI_QKV: return launch_chosen<EPI_QKV>(q, n_cu, s);
        case EPI_RESID: return launch_chosen<EPI_RESID>(q, n_cu, s);
        case EPI_SWIGLU: return launch_chosen<EPI_SWIGLU>(q, n_cu, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_mx4_call_blocked(int epi, const Mx4CallArgs &c, int n_cu, hipStream_t s) {
    if (c.n < 1 || (c.terms != 1 && c.terms != 3)) return hipErrorInvalidValue;
    const int per = 128 / c.terms;
    Mx4GemmArgs q{};
    q.w = c.w;
    q.a.in_s = c.x;
    q.a.n_rg = c.w.n_rg;
    q.a.O = c.O;
    q.ma.S = (c.n + per - 1) / per;
    q.ma.rows_last = c.n - (q.ma.S - 1) * per;
    q.ma.in_s = (int64_t)mx4_act_tiles(c.w.K) * kMx4Tile * 128;
    q.out = c.out;
    q.terms = c.terms;
    if (epi == EPI_LINEAR) return launch_chosen<EPI_LINEAR>(q, n_cu, s);
    if (epi == EPI_GATED) return launch_chosen<EPI_GATED>(q, n_cu, s);
    return hipErrorInvalidValue;
}

}  // namespace swift
