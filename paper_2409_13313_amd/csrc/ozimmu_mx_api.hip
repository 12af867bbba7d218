// C ABI of the microscaled 4-bit operators (declared in include/ozimmu_mx.h): argument checks, workspace carving and launches.
// No allocation, no host synchronisation, no state between calls.
#include "../../include/ozimmu.h"
#include "../../include/ozimmu_mx.h"
#include "ozimmu_mx.h"

namespace {

// rows <= 2^22 - 256: every grid dimension stays within the HIP limits (64 rows a workgroup along y)
constexpr int64_t MAX_ROWS = ((int64_t)1 << 22) - 256;
constexpr int64_t MAX_INNER = (int64_t)1 << 29;
constexpr int64_t MAX_LD = ((int64_t)1 << 40) - 1;
// rows x leading dimension: offsets in bytes stay within 64 bits, those of the rows that fill up a tile too (up to 2^29 rows where blocks
// lie along the columns; MAX_ROWS x MAX_LD bytes of codes or scales are below that by themselves)
constexpr int64_t MAX_SPAN = ((int64_t)1 << 60) - 1;

inline bool sizes_ok(int64_t rows, int64_t n) { return rows >= 0 && n >= 0 && rows <= MAX_ROWS && n <= MAX_INNER; }
inline bool type_ok(int type) { return type == OZIMMU_MX_F32 || type == OZIMMU_MX_BF16 || type == OZIMMU_MX_F16; }
inline bool ld_ok(int64_t ld, int64_t width) { return ld >= width && ld <= MAX_LD; }
inline bool aligned(const void* p) { return ((uintptr_t)p & 255u) == 0; }
inline bool aligned_to_type(const void* p, int type) { return ((uintptr_t)p & (type == OZIMMU_MX_F32 ? 3u : 1u)) == 0; }
inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// a packed operand of that many elements: given and aligned
int packed_status(const void* p, int64_t rows, int64_t n)
{
    if (rows == 0 || n == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return aligned(p) ? OZIMMU_OK : OZIMMU_ERR_WORKSPACE;
}
// a matrix in memory: given, aligned for its type, its rows apart
int matrix_status(int type, const void* p, int64_t rows, int64_t n, int64_t ld)
{
    if (!type_ok(type)) return OZIMMU_ERR_TYPE;
    if (!ld_ok(ld, n) || (rows > 0 && ld > MAX_SPAN / rows)) return OZIMMU_ERR_DIM;
    if (rows == 0 || n == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return aligned_to_type(p, type) ? OZIMMU_OK : OZIMMU_ERR_TYPE;
}
int workspace_status(const void* p, size_t bytes, size_t need)
{
    if (need == 0) return OZIMMU_OK;
    if (!p) return OZIMMU_ERR_NULL;
    return bytes >= need && aligned(p) ? OZIMMU_OK : OZIMMU_ERR_WORKSPACE;
}
#define CHECK(x)                             \
    do {                                     \
        const int status_ = (x);             \
        if (status_ != OZIMMU_OK) return status_; \
    } while (0)

inline int launched(hipError_t e) { return e == hipSuccess ? OZIMMU_OK : OZIMMU_ERR_HIP; }

}  // namespace

extern "C" {

size_t ozimmu_mx_bytes(int64_t rows, int64_t n) { return sizes_ok(rows, n) ? (size_t)mxl::packed_bytes(rows, n) : 0; }

int ozimmu_mx_quantize(int type, int64_t rows, int64_t n, const void* X, int64_t ldx, void* by_row, void* by_col, void* stream)
{
    if (by_row && !sizes_ok(rows, n)) return OZIMMU_ERR_DIM;
    if (by_col && !sizes_ok(n, rows)) return OZIMMU_ERR_DIM;
    if (rows < 0 || n < 0) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(type, X, rows, n, ldx));
    if (rows == 0 || n == 0) return OZIMMU_OK;
    if (!by_row && !by_col) return OZIMMU_ERR_NULL;
    if (!aligned(by_row) || !aligned(by_col)) return OZIMMU_ERR_WORKSPACE;
    return launched(mxk::launch_quantize(type, {rows, n, X, ldx, by_row, by_col}, (hipStream_t)stream));
}

int ozimmu_mx_dequantize(int type, int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, void* stream)
{
    if (!sizes_ok(rows, n)) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(type, X, rows, n, ldx));
    CHECK(packed_status(packed, rows, n));
    if (rows == 0 || n == 0) return OZIMMU_OK;
    return launched(mxk::launch_dequantize(type, rows, n, packed, X, ldx, (hipStream_t)stream));
}

static int plain_status(int64_t rows, int64_t n, const void* codes, int64_t ldc, const void* scales, int64_t lds, const void* packed)
{
    if (!sizes_ok(rows, n)) return OZIMMU_ERR_DIM;
    const int64_t blocks = (n + 31) / 32;
    if (!ld_ok(ldc, 16 * blocks) || !ld_ok(lds, blocks)) return OZIMMU_ERR_DIM;
    if (rows > 0 && n > 0 && (!codes || !scales)) return OZIMMU_ERR_NULL;
    return packed_status(packed, rows, n);
}

int ozimmu_mx_pack(int64_t rows, int64_t n, const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, void* packed,
                   void* stream)
{
    CHECK(plain_status(rows, n, codes, ldc, scales, lds, packed));
    if (rows == 0 || n == 0) return OZIMMU_OK;
    return launched(mxk::launch_pack(rows, n, codes, ldc, scales, lds, packed, (hipStream_t)stream));
}

int ozimmu_mx_unpack(int64_t rows, int64_t n, const void* packed, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                     void* stream)
{
    CHECK(plain_status(rows, n, codes, ldc, scales, lds, packed));
    if (rows == 0 || n == 0) return OZIMMU_OK;
    return launched(mxk::launch_unpack(rows, n, packed, codes, ldc, scales, lds, (hipStream_t)stream));
}

// workspace of a product whose A is quantised in the call: A packed
size_t ozimmu_mx_workspace_bytes(int64_t m, int64_t n, int64_t p)
{
    if (!sizes_ok(m, n) || !sizes_ok(p, n) || mxk::few_rows(m, p)) return 0;
    return round256((size_t)mxl::packed_bytes(m, n));
}

size_t ozimmu_mx_backward_workspace_bytes(int64_t m, int64_t n, int64_t p)
{
    // G both ways, X by columns
    if (!sizes_ok(m, p) || !sizes_ok(p, m) || !sizes_ok(n, m) || !sizes_ok(n, p)) return 0;
    return round256((size_t)(mxl::packed_bytes(m, p) + mxl::packed_bytes(p, m) + mxl::packed_bytes(n, m)));
}

int ozimmu_mx_gemm(int64_t m, int64_t n, int64_t p, float alpha, const void* A, const void* B, float beta, int type, void* D,
                   int64_t ldd, void* stream)
{
    return ozimmu_mx_gemm_way(OZIMMU_MX_WAY_AUTO, m, n, p, alpha, A, B, beta, type, D, ldd, stream);
}

int ozimmu_mx_gemm_way(int way, int64_t m, int64_t n, int64_t p, float alpha, const void* A, const void* B, float beta, int type, void* D,
                       int64_t ldd, void* stream)
{
    if (!sizes_ok(m, n) || !sizes_ok(p, n)) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(type, D, m, p, ldd));
    if (way != OZIMMU_MX_WAY_AUTO && !mxk::way_fits(way, m, n, p, ldd)) return OZIMMU_ERR_WAY;
    if (m == 0 || p == 0) return OZIMMU_OK;
    CHECK(packed_status(A, m, n));
    CHECK(packed_status(B, p, n));
    const mxk::Gemm g = {m, n, p, (const uint8_t*)A, (const uint8_t*)B, D, ldd, type, alpha, beta};
    return launched(mxk::launch_gemm(g, way, (hipStream_t)stream));
}

int ozimmu_mx_choose(int64_t m, int64_t n, int64_t p, int64_t ldd) { return mxk::choose(m, n, p, ldd); }

int ozimmu_mx_linear(int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void* X, int64_t ldx, const void* W, float beta,
                     int dtype, void* D, int64_t ldd, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!sizes_ok(m, n) || !sizes_ok(p, n)) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(xtype, X, m, n, ldx));
    CHECK(matrix_status(dtype, D, m, p, ldd));
    if (m == 0 || p == 0) return OZIMMU_OK;
    CHECK(packed_status(W, p, n));
    CHECK(workspace_status(workspace, workspace_bytes, ozimmu_mx_workspace_bytes(m, n, p)));
    const hipStream_t st = (hipStream_t)stream;
    const mxk::Gemm g = {m, n, p, (const uint8_t*)workspace, (const uint8_t*)W, D, ldd, dtype, alpha, beta};
    if (mxk::few_rows(m, p)) return launched(mxk::launch_few(g, xtype, X, ldx, st));
    if (n > 0) CHECK(launched(mxk::launch_quantize(xtype, {m, n, X, ldx, workspace, nullptr}, st)));
    return launched(mxk::launch_gemm(g, mxk::WAY_AUTO, st));
}

int ozimmu_mx_linear_backward(int64_t m, int64_t n, int64_t p, float alpha, int type, const void* G, int64_t ldg, const void* X,
                              int64_t ldx, const void* Wt, float beta_x, int dx_type, void* dX, int64_t lddx, float beta_w,
                              int dw_type, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!sizes_ok(m, p) || !sizes_ok(p, m) || !sizes_ok(n, m) || !sizes_ok(n, p)) return OZIMMU_ERR_DIM;
    CHECK(matrix_status(type, G, m, p, ldg));
    if (dX) {
        CHECK(matrix_status(dx_type, dX, m, n, lddx));
        CHECK(packed_status(Wt, n, p));
    }
    if (dW) {
        CHECK(matrix_status(type, X, m, n, ldx));
        CHECK(matrix_status(dw_type, dW, p, n, lddw));
    }
    CHECK(workspace_status(workspace, workspace_bytes, ozimmu_mx_backward_workspace_bytes(m, n, p)));
    const hipStream_t st = (hipStream_t)stream;
    uint8_t* const g_rows = (uint8_t*)workspace;
    uint8_t* const g_cols = g_rows + mxl::packed_bytes(m, p);
    uint8_t* const x_cols = g_cols + mxl::packed_bytes(p, m);
    const bool want_x = dX && m > 0 && n > 0, want_w = dW && p > 0 && n > 0;
    if (m > 0 && p > 0) {
        const mxk::Quantize gq = {m, p, G, ldg, want_x ? g_rows : nullptr, want_w ? g_cols : nullptr}, xq = {m, n, X, ldx, nullptr, x_cols};
        if (want_w)
            CHECK(launched(mxk::launch_quantize2(type, gq, xq, st)));
        else if (want_x)
            CHECK(launched(mxk::launch_quantize(type, gq, st)));
    }
    const mxk::Gemm gx = {m, p, n, g_rows, (const uint8_t*)Wt, dX, lddx, dx_type, alpha, beta_x};
    const mxk::Gemm gw = {p, m, n, g_cols, x_cols, dW, lddw, dw_type, alpha, beta_w, true};
    if (want_x && want_w) return launched(mxk::launch_gemm2(gx, gw, st));
    if (want_x) return launched(mxk::launch_gemm(gx, mxk::WAY_AUTO, st));
    if (want_w) return launched(mxk::launch_gemm(gw, mxk::WAY_AUTO, st));
    return OZIMMU_OK;
}

}  // extern "C"
