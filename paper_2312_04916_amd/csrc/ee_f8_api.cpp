// Host side of products with weights held in 8 bits (ee_f8_* of ee.h): argument checks.
#include "ee_f8.h"
#include "ee_internal.h"

using namespace ee;

namespace {

int check_shape(int n, int k) { return n < 1 || n > (1 << 22) || k < 1 || k > (1 << 18) ? EE_ERR_CONFIG : EE_OK; }
bool is_type(int dtype) { return dtype == EE_F32 || dtype == EE_BF16; }
int64_t size_of(int dtype) { return dtype == EE_BF16 ? 2 : 4; }
int hip_status(hipError_t e) { return e == hipSuccess ? EE_OK : ee::note_hip_error((int)e); }

// Rows of `width` bytes that lie `stride` bytes apart, from the lowest on, or one piece of memory.
struct Rows {
    uintptr_t lo;
    int64_t rows, stride, width;
    Rows(const void* p, int n, int64_t elements_apart, int cols, int dtype)
        : rows(n), stride((elements_apart < 0 ? -elements_apart : elements_apart) * size_of(dtype)), width(cols * size_of(dtype)) {
        lo = (uintptr_t)p - (uintptr_t)(elements_apart < 0 ? (rows - 1) * stride : 0);
        if (stride == 0) rows = 1;
    }
    Rows(const void* p, size_t bytes) : lo((uintptr_t)p), rows(1), stride(0), width((int64_t)bytes) {}
    uintptr_t hi() const { return lo + (uintptr_t)((rows - 1) * stride + width); }
    // Whether any byte is in both, where the strides are the same and no row reaches into the next (columns of one buffer); elsewhere
    // whether the ranges that they span meet.
    bool overlaps(const Rows& o) const {
        if (hi() <= o.lo || o.hi() <= lo) return false;
        const int64_t s = rows > 1 ? stride : o.stride;
        if ((rows == 1 && o.rows == 1) || (o.rows > 1 && o.stride != s) || width > s || o.width > s) return true;
        // o's first row begins `in` bytes behind the beginning of this one's row `at`, which there may be or not
        const int64_t d = (int64_t)(o.lo - lo), at = d >= 0 ? d / s : -((s - 1 - d) / s), in = d - at * s;
        auto some_of = [&](int64_t row) { return row < rows && row > -o.rows; };  // o's rows from here on: any beside one of these
        return (in < width && some_of(at)) || (in + o.width > s && some_of(at + 1));
    }
};

}  // namespace

extern "C" {

int ee_f8_bytes(int n, int k, int pair, size_t* weight_bytes) {
    if (!weight_bytes) return EE_ERR_ARG;
    const int rc = check_shape(n, k);
    if (rc != EE_OK) return rc;
    *weight_bytes = F8Shape{n, k, pair != 0}.bytes();
    return EE_OK;
}

int ee_f8_pack(int n, int k, int pair, int dtype, const void* dev_w, int64_t w_row_stride, const void* dev_up, int64_t up_row_stride,
               void* dev_weight, size_t weight_bytes, void* stream) {
    int rc = check_shape(n, k);
    if (rc != EE_OK) return rc;
    if (!is_type(dtype)) return EE_ERR_CONFIG;
    if (!dev_w || !dev_weight || (pair != 0) != (dev_up != nullptr) || (uintptr_t)dev_weight & 255) return EE_ERR_ARG;
    if (((uintptr_t)dev_w | (uintptr_t)dev_up) & (size_of(dtype) - 1)) return EE_ERR_ARG;
    const F8Shape s{n, k, pair != 0};
    if (weight_bytes < s.bytes()) return EE_ERR_NOMEM;
    const Rows out(dev_weight, s.bytes());
    if (out.overlaps(Rows(dev_w, n, w_row_stride, k, dtype)) || (pair && out.overlaps(Rows(dev_up, n, up_row_stride, k, dtype)))) return EE_ERR_ARG;
    return hip_status(launch_f8_pack(s, dtype, dev_w, w_row_stride, dev_up, up_row_stride, (char*)dev_weight, (hipStream_t)stream));
}

int ee_f8_unpack(int n, int k, int pair, int up, const void* dev_weight, int dtype, void* dev_w, void* stream) {
    int rc = check_shape(n, k);
    if (rc != EE_OK) return rc;
    if (!is_type(dtype)) return EE_ERR_CONFIG;
    if (!dev_w || !dev_weight || (up && !pair) || (uintptr_t)dev_weight & 255 || (uintptr_t)dev_w & (size_of(dtype) - 1)) return EE_ERR_ARG;
    const F8Shape s{n, k, pair != 0};
    if (Rows(dev_weight, s.bytes()).overlaps(Rows(dev_w, n, k, k, dtype))) return EE_ERR_ARG;
    return hip_status(launch_f8_unpack(s, up != 0, (const char*)dev_weight, dtype, dev_w, (hipStream_t)stream));
}

int ee_f8_matmul_bytes(int m, int n, int k, int pair, int y_dtype, size_t* workspace_bytes) {
    if (!workspace_bytes || m < 0 || m > (1 << 20)) return EE_ERR_ARG;
    const int rc = check_shape(n, k);
    if (rc != EE_OK) return rc;
    if (!is_type(y_dtype)) return EE_ERR_CONFIG;
    *workspace_bytes = f8_workspace(m, n, k, pair != 0, y_dtype);
    return EE_OK;
}

int ee_debug_f8_launch(int m, int n, int k, int pair, int32_t shape[4]) {
    if (!shape || m < 1 || m > (1 << 20)) return EE_ERR_ARG;
    const int rc = check_shape(n, k);
    if (rc != EE_OK) return rc;
    f8_launch_shape(m, n, k, pair != 0, shape);
    return EE_OK;
}

int ee_f8_matmul(int m, int n, int k, int pair, const void* dev_weight, int x_dtype, const void* dev_x, int64_t x_row_stride, int y_dtype,
                 void* dev_y, int64_t y_row_stride, const void* dev_add, int64_t add_row_stride, void* dev_workspace,
                 size_t workspace_bytes, void* stream) {
    size_t need;
    const int rc = ee_f8_matmul_bytes(m, n, k, pair, y_dtype, &need);
    if (rc != EE_OK) return rc;
    if (!is_type(x_dtype)) return EE_ERR_CONFIG;
    if (m == 0) return EE_OK;
    const int64_t xs = size_of(x_dtype), ys = size_of(y_dtype);
    if (!dev_weight || !dev_x || !dev_y || (uintptr_t)dev_weight & 255 || (uintptr_t)dev_x & (xs - 1) || ((uintptr_t)dev_y | (uintptr_t)dev_add) & (ys - 1))
        return EE_ERR_ARG;
    // rows of y must not fall into one another, and x, the weight and the workspace are read while results are written
    if (m > 1 && (y_row_stride < 0 ? -y_row_stride : y_row_stride) < n) return EE_ERR_ARG;
    const F8Shape s{n, k, pair != 0};
    const Rows y(dev_y, m, y_row_stride, n, y_dtype), x(dev_x, m, x_row_stride, k, x_dtype), add(dev_add, m, add_row_stride, n, y_dtype);
    const Rows work(dev_workspace, need), weight(dev_weight, s.bytes());
    if (y.overlaps(x) || y.overlaps(weight)) return EE_ERR_ARG;
    if (dev_add && y.overlaps(add) && !(dev_add == dev_y && (m == 1 || add_row_stride == y_row_stride))) return EE_ERR_ARG;
    if (workspace_bytes < need) return EE_ERR_NOMEM;
    if (need && (!dev_workspace || (uintptr_t)dev_workspace & 255 || work.overlaps(y) || work.overlaps(x) || work.overlaps(weight) || (dev_add && work.overlaps(add))))
        return EE_ERR_ARG;
    F8Product p;
    p.m = m, p.n = n, p.k = k, p.pair = pair != 0;
    p.weight = (const char*)dev_weight;
    p.x = dev_x, p.x_dtype = x_dtype, p.x_row = x_row_stride;
    p.y = dev_y, p.y_dtype = y_dtype, p.y_row = y_row_stride;
    p.add = dev_add, p.add_row = add_row_stride;
    p.workspace = (char*)dev_workspace;
    return hip_status(launch_f8_matmul(p, (hipStream_t)stream));
}

}  // extern "C"
