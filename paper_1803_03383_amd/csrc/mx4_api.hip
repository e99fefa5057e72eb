// C ABI of the MX4 operators: argument checks.
#include "halp_internal.hpp"
#include "mx4.hpp"

using namespace halp;

namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
constexpr int64_t kMost = int64_t(1) << 31;

// A launch holds fewer than 2^32 threads.  A product's tiles have 2 threads for each of their 64, 128 or 256 rows; A by B
// tiles of 64 are at most (A + 1) / 2 by (B + 1) / 2 of 128 and (A + 3) / 4 by (B + 3) / 4 of 256, and with A = 1, where
// these weigh most, 512 (B + 3) / 4 < 2^32 where B < 2^25 - 3.
bool too_many_tiles(int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 63) / 64) >= (int64_t(1) << 25) - 3; }

int check_matrix(const halp_mx4& q) {
  if (q.rows < 0 || q.cols < 0 || q.rows >= kMost || q.cols >= (int64_t(1) << 24)) return HALP_ERR_INVALID;
  if (q.rows == 0 || q.cols == 0) return HALP_OK;  // nothing is stored
  if (!q.codes || !q.scales) return HALP_ERR_NULL;
  if (q.ldc < 64 * mx_groups(q.cols) || q.lds < 4 * mx_groups(q.cols)) return HALP_ERR_INVALID;
  if (q.ldc >= (1 << 23) || q.lds >= (1 << 23)) return HALP_ERR_INVALID;  // a tile's rows are within 32 bits
  if (q.ldc % 16 || q.lds % 4 || !aligned(q.codes, 16) || !aligned(q.scales, 4)) return HALP_ERR_ALIGN;
  return HALP_OK;
}

// rows x cols elements of `type` with ld elements from row to row
int check_plain(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ld) {
  if (!type_known(type) || rows < 0 || cols < 0 || rows >= kMost || cols >= kMost) return HALP_ERR_INVALID;
  if (rows == 0 || cols == 0) return HALP_OK;
  if (!x) return HALP_ERR_NULL;
  if (ld < cols || ld >= (int64_t(1) << 40)) return HALP_ERR_INVALID;
  return aligned(x, type_bytes(type)) ? HALP_OK : HALP_ERR_ALIGN;
}

// compute units of the current device
int count_cus(int* cus) {
  int dev = 0;
  if (hip_fail(hipGetDevice(&dev), "hipGetDevice") ||
      hip_fail(hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev), "hipDeviceGetAttribute"))
    return HALP_ERR_HIP;
  return HALP_OK;
}

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int halp_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const halp_mx4* q,
                      const halp_mx4* qt, int32_t rounding, uint64_t seed, int64_t epoch, void* stream) {
  if (!q && !qt) return HALP_ERR_NULL;
  int rc = check_plain(x, type, rows, cols, ldx);
  if (rc != HALP_OK) return rc;
  if (rounding != HALP_ROUND_NEAREST && rounding != HALP_ROUND_STOCHASTIC) return HALP_ERR_INVALID;
  if (epoch < 0 || epoch >= (int64_t(1) << 32)) return HALP_ERR_INVALID;
  if (q && (q->rows != rows || q->cols != cols)) return HALP_ERR_INVALID;
  if (qt && (qt->rows != cols || qt->cols != rows)) return HALP_ERR_INVALID;
  if (q && (rc = check_matrix(*q)) != HALP_OK) return rc;
  if (qt && (rc = check_matrix(*qt)) != HALP_OK) return rc;
  if (rows == 0 || cols == 0) return HALP_OK;
  MxView v, vt;
  if (q) v = mx_view(*q);
  if (qt) vt = mx_view(*qt);
  int cus = 0;
  if ((rc = count_cus(&cus)) != HALP_OK) return rc;
  return launch_mx4_quantize(x, type, rows, cols, ldx, q ? &v : nullptr, qt ? &vt : nullptr, rounding, seed,
                             (uint32_t)epoch, cus, as_stream(stream));
}

int halp_mx4_dequantize(const halp_mx4* q, void* out, int32_t type, int64_t ldo, void* stream) {
  if (!q) return HALP_ERR_NULL;
  int rc = check_matrix(*q);
  if (rc == HALP_OK) rc = check_plain(out, type, q->rows, q->cols, ldo);
  if (rc != HALP_OK || q->rows == 0 || q->cols == 0) return rc;
  return launch_mx4_dequantize(mx_view(*q), out, type, ldo, as_stream(stream));
}

int halp_mx4_product(const halp_mx4* a, const halp_mx4* b, void* c, int32_t type, int64_t ldc, int32_t accumulate,
                     void* workspace, int64_t workspace_bytes, void* stream) {
  if (!a || !b) return HALP_ERR_NULL;
  int rc = check_matrix(*a);
  if (rc == HALP_OK) rc = check_matrix(*b);
  if (rc == HALP_OK) rc = check_plain(c, type, a->rows, b->rows, ldc);
  if (rc != HALP_OK) return rc;
  if (a->cols != b->cols || (accumulate != 0 && accumulate != 1) || workspace_bytes < 0) return HALP_ERR_INVALID;
  if (accumulate && type != HALP_TYPE_F32) return HALP_ERR_UNSUPPORTED;
  if (workspace && !aligned(workspace, 16)) return HALP_ERR_ALIGN;
  if (too_many_tiles(a->rows, b->rows)) return HALP_ERR_UNSUPPORTED;
  if (a->rows == 0 || b->rows == 0) return HALP_OK;
  int cus = 0;
  if ((rc = count_cus(&cus)) != HALP_OK) return rc;
  return launch_mx4_product(mx_view(*a), mx_view(*b), c, type, ldc, accumulate != 0, workspace,
                            workspace ? workspace_bytes : 0, cus, as_stream(stream));
}

int halp_mx4_product_workspace(int64_t M, int64_t N, int64_t K, int64_t* bytes) {
  if (!bytes) return HALP_ERR_NULL;
  if (M < 0 || N < 0 || K < 0 || M >= kMost || N >= kMost || K >= kMost) return HALP_ERR_INVALID;
  if (too_many_tiles(M, N)) return HALP_ERR_UNSUPPORTED;
  int cus = 0;
  if (const int rc = count_cus(&cus)) return rc;
  *bytes = mx4_product_workspace(M, N, K, cus);
  return HALP_OK;
}

int halp_mx4_row_product(const void* x, int32_t xtype, int64_t M, int64_t ldx, const halp_mx4* w, void* y,
                         int32_t ytype, int64_t ldy, void* stream) {
  if (!w) return HALP_ERR_NULL;
  int rc = check_matrix(*w);
  if (rc == HALP_OK) rc = check_plain(x, xtype, M, w->cols, ldx);
  if (rc == HALP_OK) rc = check_plain(y, ytype, M, w->rows, ldy);
  if (rc != HALP_OK) return rc;
  if (M > 16 || w->cols > kMxRowMost) return HALP_ERR_UNSUPPORTED;
  if (M == 0 || w->rows == 0) return HALP_OK;
  int cus = 0;
  if ((rc = count_cus(&cus)) != HALP_OK) return rc;
  return launch_mx4_row_product(x, xtype, M, ldx, mx_view(*w), y, ytype, ldy, cus, as_stream(stream));
}

}  // extern "C"
