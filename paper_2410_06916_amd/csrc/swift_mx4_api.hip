// C-ABI layer of the MXFP4 operators (declared in include/swift.h): checks of arguments, sizes, and the launches a call is made of.
#include <algorithm>
#include <atomic>

#include "swift_mx4.h"

using namespace swift;

namespace {

constexpr int kMaxSide = 1 << 22;  // rows and depth of a packed matrix

int device_status(hipError_t e, const char *what) {
    return e == hipSuccess ? SWIFT_OK : api_fail(SWIFT_EDEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

int check_matrix(int rows, int depth) {
    if (rows < 1 || depth < 1 || rows > kMaxSide || depth > kMaxSide)
        return api_fail(SWIFT_EINVAL, "a packed matrix has 1 to 2^22 rows and a depth of 1 to 2^22");
    return SWIFT_OK;
}
bool known_dtype(int t) { return t == SWIFT_F32 || t == SWIFT_BF16; }
bool aligned(const void *p, int dtype) { return ((uintptr_t)p & (dtype == SWIFT_F32 ? 3 : 1)) == 0; }

int row_groups(int rows, bool gated) { return gated ? (rows + 7) / 8 : (rows + 15) / 16; }
Mx4Matrix matrix_at(const void *packed, int rows, int depth, bool gated) {
    const int n_rg = row_groups(rows, gated);
    const auto *codes = (const uint8_t *)packed;
    return Mx4Matrix{codes, codes + mx4_code_bytes(n_rg, depth), depth, mx4_tiles(depth), n_rg};
}

int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 256;
    std::atomic<int> *at = dev >= 0 && dev < 64 ? &known[dev] : nullptr;
    if (at && (n = at->load(std::memory_order_relaxed)) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) n = 256;
    if (at) at->store(n, std::memory_order_relaxed);
    return n;
}

// Rows of a blocked launch (a multiple of both sub-block heights): bounds the workspace.
constexpr int kBlockedRows = 128 * 42;

bool few(int n, int x_dtype) { return n <= kMx4FewColumns / mx4_terms(x_dtype); }
// Of a product's workspace, what the rows as columns take, and the slices' sums behind them.
uint64_t activation_bytes(int depth, int n, int x_dtype) {
    const uint64_t terms = mx4_terms(x_dtype);
    if (mx4_rows_x32(x_dtype, n, depth)) return 0;
    if (few(n, x_dtype)) return (uint64_t)mx4_tiles(depth) * kMx4Tile * 2 * mx4_pitch((int)terms * n);
    const uint64_t k = (uint64_t)mx4_act_tiles(depth) * kMx4Tile * 2;
    const int per = 128 / (int)terms, rows = std::min(n, kBlockedRows);
    return k * 128 * ((rows + per - 1) / per);
}
uint64_t part_bytes(int rows, int depth, bool gated, int n, int x_dtype) {
    if (gated || !few(n, x_dtype) || mx4_rows_x32(x_dtype, n, depth)) return 0;
    const int NC = mx4_terms(x_dtype) * n, n_rg = row_groups(rows, false);
    return mx4_sliced(NC, n_rg, mx4_tiles(depth)) ? mx4_part_bytes(NC, n_rg) : 0;
}
uint64_t workspace(int rows, int depth, bool gated, int n, int x_dtype) {
    return activation_bytes(depth, n, x_dtype) + part_bytes(rows, depth, gated, n, x_dtype);
}

struct Call {
    void *y;
    int y_dtype;
    int64_t ld_y;
    const void *x;
    int x_dtype;
    int64_t ld_x;
    const void *packed;
    int rows, depth, n;
    const void *residual;
    int64_t ld_res;
    void *ws;
    uint64_t ws_bytes;
};

int product(int epi, const Call &c, void *stream) {
    if (int rc = check_matrix(c.rows, c.depth)) return rc;
    if (c.n < 0) return api_fail(SWIFT_EINVAL, "a negative number of rows");
    if (!known_dtype(c.x_dtype) || !known_dtype(c.y_dtype)) return api_fail(SWIFT_EINVAL, "unknown dtype");
    if (c.n == 0) return SWIFT_OK;
    if (!c.y || !c.x || !c.packed) return api_fail(SWIFT_EINVAL, "null argument");
    if (c.ld_x < c.depth || c.ld_y < c.rows || (c.residual && c.ld_res < c.rows)) return api_fail(SWIFT_EINVAL, "rows overlap: a leading dimension is too small");
    if (!aligned(c.x, c.x_dtype) || !aligned(c.y, c.y_dtype) || (c.residual && !aligned(c.residual, c.y_dtype)) || ((uintptr_t)c.packed & 255))
        return api_fail(SWIFT_EINVAL, "a pointer is not aligned to its elements (a packed matrix: to 256 bytes)");
    const uint64_t need = workspace(c.rows, c.depth, epi == EPI_GATED, c.n, c.x_dtype);
    if (need && (!c.ws || ((uintptr_t)c.ws & 255) || c.ws_bytes < need))
        return api_fail(SWIFT_ECAPACITY, "the workspace is missing, not aligned to 256 bytes, or smaller than swift_mx4_workspace says");
    const auto s = (hipStream_t)stream;
    const int terms = mx4_terms(c.x_dtype), xb = c.x_dtype == SWIFT_F32 ? 4 : 2, yb = c.y_dtype == SWIFT_F32 ? 4 : 2;
    const bool blocked = !few(c.n, c.x_dtype);
    Mx4CallArgs a{};
    a.w = matrix_at(c.packed, c.rows, c.depth, epi == EPI_GATED);
    a.x = (const uint16_t *)c.ws;
    a.terms = terms;
    a.O = c.rows;
    a.part = part_bytes(c.rows, c.depth, epi == EPI_GATED, c.n, c.x_dtype) ? (float *)((char *)c.ws + activation_bytes(c.depth, c.n, c.x_dtype)) : nullptr;
    if (!blocked && (mx4_rows_x32(c.x_dtype, c.n, c.depth) || mx4_rows_direct(c.x, c.x_dtype, c.ld_x, c.n, c.depth))) {
        a.n = c.n;
        a.direct = c.x_dtype == SWIFT_BF16;
        a.x = a.direct ? (const uint16_t *)c.x : nullptr;
        a.x32 = a.direct ? nullptr : (const float *)c.x;
        a.ld_x = c.ld_x;
        a.out = Mx4Out{c.y, c.y_dtype, c.ld_y, c.residual, c.ld_res};
        return device_status(launch_mx4_call(epi, a, compute_units(), s), "MXFP4 product");
    }
    for (int64_t r0 = 0; r0 < c.n; r0 += kBlockedRows) {
        a.n = (int)std::min<int64_t>(kBlockedRows, c.n - r0);
        const char *x = (const char *)c.x + r0 * c.ld_x * xb;
        const Mx4ActArgs act = blocked ? Mx4ActArgs{x, c.x_dtype, c.ld_x, a.n, c.depth, mx4_act_tiles(c.depth), 128 / terms, 128, (uint16_t *)c.ws}
                                       : Mx4ActArgs{x, c.x_dtype, c.ld_x, a.n, c.depth, a.w.S, a.n, mx4_pitch(terms * a.n), (uint16_t *)c.ws};
        if (int rc = device_status(launch_mx4_activations(act, s), "activations of an MXFP4 product")) return rc;
        a.out = Mx4Out{(char *)c.y + r0 * c.ld_y * yb, c.y_dtype, c.ld_y, c.residual ? (const char *)c.residual + r0 * c.ld_res * yb : nullptr, c.ld_res};
        const hipError_t e = blocked ? launch_mx4_call_blocked(epi, a, compute_units(), s) : launch_mx4_call(epi, a, compute_units(), s);
        if (int rc = device_status(e, "MXFP4 product")) return rc;
    }
    return SWIFT_OK;
}

}  // namespace

extern "C" int swift_mx4_bytes(int rows, int depth, int gated, uint64_t *bytes) {
    if (!bytes) return api_fail(SWIFT_EINVAL, "null output");
    if (int rc = check_matrix(rows, depth)) return rc;
    const int n_rg = row_groups(rows, gated != 0);
    *bytes = mx4_code_bytes(n_rg, depth) + mx4_scale_bytes(n_rg, depth);
    return SWIFT_OK;
}

extern "C" int swift_mx4_workspace(int rows, int depth, int gated, int n, int x_dtype, uint64_t *bytes) {
    if (!bytes) return api_fail(SWIFT_EINVAL, "null output");
    if (int rc = check_matrix(rows, depth)) return rc;
    if (n < 0 || !known_dtype(x_dtype)) return api_fail(SWIFT_EINVAL, "bad argument");
    *bytes = workspace(rows, depth, gated != 0, n, x_dtype);
    return SWIFT_OK;
}

extern "C" int swift_mx4_quantize(void *packed, const void *w, int64_t ld_w, const void *up, int64_t ld_up, int dtype, int rows, int depth,
                                  void *stream) {
    if (!packed || !w) return api_fail(SWIFT_EINVAL, "null argument");
    if (int rc = check_matrix(rows, depth)) return rc;
    if (!known_dtype(dtype)) return api_fail(SWIFT_EINVAL, "unknown dtype");
    if (ld_w < depth || (up && ld_up < depth)) return api_fail(SWIFT_EINVAL, "rows overlap: a leading dimension is too small");
    if (((uintptr_t)packed & 255) || !aligned(w, dtype) || (up && !aligned(up, dtype)))
        return api_fail(SWIFT_EINVAL, "a pointer is not aligned to its elements (a packed matrix: to 256 bytes)");
    const Mx4Matrix m = matrix_at(packed, rows, depth, up != nullptr);
    const Mx4QuantArgs a{w, up, dtype, ld_w, ld_up, rows, depth, (uint8_t *)m.codes, (uint8_t *)m.scales, m.n_rg, up ? TILE_GATEUP : TILE_PLAIN, 0};
    return device_status(launch_mx4_quantize(a, (hipStream_t)stream), "swift_mx4_quantize");
}

extern "C" int swift_mx4_dequantize(void *w, int64_t ld_w, int dtype, const void *packed, int rows, int depth, int gated, void *stream) {
    if (!packed || !w) return api_fail(SWIFT_EINVAL, "null argument");
    if (int rc = check_matrix(rows, depth)) return rc;
    if (!known_dtype(dtype)) return api_fail(SWIFT_EINVAL, "unknown dtype");
    if (ld_w < depth) return api_fail(SWIFT_EINVAL, "rows overlap: a leading dimension is too small");
    if (((uintptr_t)packed & 255) || !aligned(w, dtype))
        return api_fail(SWIFT_EINVAL, "a pointer is not aligned to its elements (a packed matrix: to 256 bytes)");
    Mx4DequantArgs a{matrix_at(packed, rows, depth, gated != 0), w, dtype, ld_w, rows, depth, gated ? TILE_GATEUP : TILE_PLAIN, 0};
    return device_status(launch_mx4_dequantize(a, (hipStream_t)stream), "swift_mx4_dequantize");
}

extern "C" int swift_mx4_linear(void *y, int64_t ld_y, int y_dtype, const void *x, int64_t ld_x, int x_dtype, int n, const void *packed, int rows,
                                int depth, const void *residual, int64_t ld_residual, void *workspace, uint64_t workspace_bytes, void *stream) {
    return product(EPI_LINEAR, Call{y, y_dtype, ld_y, x, x_dtype, ld_x, packed, rows, depth, n, residual, ld_residual, workspace, workspace_bytes}, stream);
}

extern "C" int swift_mx4_swiglu(void *h, int64_t ld_h, int h_dtype, const void *x, int64_t ld_x, int x_dtype, int n, const void *packed, int rows,
                                int depth, void *workspace, uint64_t workspace_bytes, void *stream) {
    return product(EPI_GATED, Call{h, h_dtype, ld_h, x, x_dtype, ld_x, packed, rows, depth, n, nullptr, 0, workspace, workspace_bytes}, stream);
}
