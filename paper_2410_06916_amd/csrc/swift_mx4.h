// MXFP4 matrices: launch interface between the C-ABI layers and the kernels of swift_mx4_pack.hip and swift_mx4.hip.
//
// The format (OCP Microscaling Formats v1.0): 32 consecutive weights of a row share the scale 2^(e - 127), e one byte; an element is
// four bits, a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  e = 255: the block is NaN.  A row's last block holds what is left of it.
//
// A packed matrix [O][K] is a plane of codes and a plane of scales behind it, both cut into pieces of 16 rows (a row group, rows as
// TileMode says) x 128 k (a super-tile), piece (rg, s) at number rg S + s, S = ceil(K / 128):
//   codes   1 KB: lane l = 16 kg + j of a wavefront owns the 16 bytes of one block, tile row j, k = 128 s + 32 kg .. + 31, the
//           earlier weight of a byte in its low half;
//   scales  64 bytes: lane l's is that block's.
// So one 128-bit load per lane is a whole block with one scale, and word t of it (k = 32 kg + 8 t ..) is, converted, the A operand of the
// t-th of four v_mfma_f32_16x16x32_bf16, whose B operand lane (kg, column) then holds k = 128 s + 32 kg + 8 t .. + 7: the reduction index
// is permuted within 128 on both sides alike, which costs nothing.  Rows and k past the matrix are zero codes.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "swift_kernels.h"

namespace swift {

constexpr int kMx4Block = 32, kMx4Tile = 128;
__host__ __device__ inline int mx4_tiles(int K) { return (K + kMx4Tile - 1) / kMx4Tile; }
inline uint64_t mx4_code_bytes(uint64_t n_rg, int K) { return n_rg * mx4_tiles(K) * 1024; }
inline uint64_t mx4_scale_bytes(uint64_t n_rg, int K) { return n_rg * mx4_tiles(K) * 64; }

struct Mx4Matrix {
    const uint8_t *codes, *scales;
    int K, S;   // depth, super-tiles of a row group
    int n_rg;   // row groups
};

// ---- packing (swift_mx4_pack.hip)
struct Mx4QuantArgs {
    const void *src, *up;  // [src_rows][K], rows ld and ld_up elements apart; TILE_GATEUP: the gate and the up rows (nullptr: left as they are)
    int dtype;             // F32 or BF16
    int64_t ld, ld_up;
    int src_rows, K;
    uint8_t *codes, *scales;  // first row group written
    int n_rg, mode, head_dim;  // as in TileArgs
};
hipError_t launch_mx4_quantize(const Mx4QuantArgs &a, hipStream_t s);

struct Mx4DequantArgs {
    Mx4Matrix w;
    void *dst;  // [rows][K] (TILE_GATEUP: the gate rows, then the up rows), rows ld elements apart
    int dtype;
    int64_t ld;
    int rows, K, mode;  // rows: of the matrix (TILE_GATEUP: of each half); TILE_PLAIN or TILE_GATEUP
    int row0;           // set by the launcher: row of the launch's first row group
};
hipError_t launch_mx4_dequantize(const Mx4DequantArgs &a, hipStream_t s);

// Super-tiles of activations that the blocked product reads: its pipeline has at least two.
__host__ __device__ inline int mx4_act_tiles(int K) { return K > kMx4Tile ? mx4_tiles(K) : 2; }
// Activations [n][K] to the B operand's layout, in sub-blocks of `per` rows: [sub-block][16 S chunks][pitch columns][8 k] bf16, zeros past
// K; a bf16 row is one column, an fp32 row three (value = hi + mid + lo; column 3 r + term).  Columns of rows that do not exist
// are left as they are.
inline int mx4_terms(int dtype) { return dtype == F32 ? 3 : 1; }
struct Mx4ActArgs {
    const void *x;
    int dtype;
    int64_t ld;
    int n, K, S;
    int per, pitch;
    uint16_t *out;
};
hipError_t launch_mx4_activations(const Mx4ActArgs &a, hipStream_t s);

// Columns from one chunk to the next for a launch of few rows: whole lines of 128 bytes, where there is more than one column block to read.
inline int mx4_pitch(int columns) { return columns <= 16 ? columns : (columns + 7) / 8 * 8; }

// ---- products (swift_mx4.hip; blocked: swift_mx4_gemm.hip)
// What follows the dot products of a call that is not part of a model's pass, beside Epilogue's.
enum Mx4Epilogue : int {
    EPI_LINEAR = 8,  // y = W x (+ residual)
    EPI_GATED = 9,   // h = silu(gate) * up
};
struct Mx4Out {
    void *y;
    int dtype;
    int64_t ld;
    const void *residual;  // nullptr, or of y's type
    int64_t ld_res;
};
// Up to this many columns a call's product goes through the kernels that read every weight once for all rows, beyond through the
// blocked one.
constexpr int kMx4FewColumns = 96;

// A model's projection (epilogue: EPI_QKV, EPI_RESID or EPI_SWIGLU) of a block of a.R rows, as launch_mv, over the row groups [rg0, a.n_rg) of w.
// part: mx4_part_bytes(kMx4FewColumns, kMx4SlicedGroups).
hipError_t launch_mx4_mv(int epilogue, const MvArgs &a, const Mx4Matrix &w, int rg0, int n_cu, float *part, hipStream_t s);
// A call's product: n rows (at most kMx4FewColumns columns) against w, O results a row (EPI_GATED: of the gate and the up half each).
// The rows: as launch_mx4_activations lays them out (one sub-block, pitch mx4_pitch); or as the caller has them, bf16 (direct:
// rows of 16-byte units, mx4_rows_direct) or fp32 (x32: mx4_rows_x32), ld_x elements apart.
struct Mx4CallArgs {
    Mx4Matrix w;
    const uint16_t *x;
    int n, terms, O;
    Mx4Out out;
    bool direct;
    const float *x32;
    int64_t ld_x;
    float *part;  // for slices (mx4_sliced)
};
// LDS that the eight slices of B take there: each 16 bytes of zeros and its lines (columns chunk by chunk, chunk_bytes a chunk), 16 bytes apart.
__host__ __device__ inline uint32_t mx4_lds_line(int slice_tiles, uint32_t chunk_bytes) { return 16u * slice_tiles * chunk_bytes + 16; }
inline size_t mx4_lds_bytes(int K, int lines, int chunk_bytes) { return 8 * (16 + (size_t)lines * mx4_lds_line((mx4_tiles(K) + 7) / 8, chunk_bytes)); }
constexpr size_t kMx4LdsMost = 96 * 1024;
// (few enough for one column block, and for LDS: more rows are read more often, and are worth laying out first)
inline bool mx4_rows_direct(const void *x, int dtype, int64_t ld, int n, int K) {
    return dtype == BF16 && ((uintptr_t)x & 15) == 0 && (K & 7) == 0 && n <= 16 && (n == 1 || ((ld & 7) == 0 && ld < 1 << 24)) &&
           mx4_lds_bytes(K, n, 16) <= kMx4LdsMost;
}
// (three columns a row in one column block, and their terms in LDS)
inline bool mx4_rows_x32(int dtype, int n, int K) { return dtype == F32 && n <= 5 && mx4_lds_bytes(K, 1, 48 * n) <= kMx4LdsMost; }
hipError_t launch_mx4_call(int epilogue, const Mx4CallArgs &a, int n_cu, hipStream_t s);

// Columns in memory for B: NC of them, from x, b_col bytes from one to the next, b_chunk from one chunk of eight k to the next, `bytes` in all.
struct Mx4Columns {
    const void *x;
    int NC;
    uint32_t bytes, b_col, b_chunk;
};
// Up to 96 columns (b_col 16, NT a row) in the same order of sums as launch_mx4_mv and launch_mx4_call (swift_mx4_narrow.hip).  A wide matrix:
// a model's gate and up (EPI_SWIGLU, a) or a call's (a.R, a.O, a.n_rg and out).
hipError_t launch_mx4_narrow(int epilogue, const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, const Mx4Columns &c, int NT, int n_cu, hipStream_t s);
// A deep one with few rows, the slices of its depth in workgroups of their own: EPI_RESID of a model or EPI_LINEAR of a call.  part:
// mx4_part_bytes.
constexpr int kMx4SlicedGroups = 768;
inline bool mx4_sliced(int NC, int n_rg, int S) { return NC > 16 && NC <= kMx4FewColumns && n_rg <= kMx4SlicedGroups && S > 64; }
constexpr uint64_t mx4_part_bytes(int NC, int n_rg) { return (uint64_t)8 * n_rg * NC * 64; }
hipError_t launch_mx4_slices(int epilogue, const Mx4Matrix &w, const MvArgs &a, const Mx4Out &out, const Mx4Columns &c, int NT, float *part, hipStream_t s);

// A prompt macro block of a model, as launch_gemm, over the row groups [rg0, a.n_rg) of w.  The activations of a sub-block are
// mx4_act_tiles(K) super-tiles, zeros past K.
hipError_t launch_mx4_macro(int epilogue, const MvArgs &a, const MacroArgs &ma, const Mx4Matrix &w, int rg0, int n_cu, hipStream_t s);
// A call's product of any number of rows, in sub-blocks of 128 / terms rows and 128 columns, mx4_act_tiles(K) super-tiles each.
hipError_t launch_mx4_call_blocked(int epilogue, const Mx4CallArgs &a, int n_cu, hipStream_t s);

}  // namespace swift
