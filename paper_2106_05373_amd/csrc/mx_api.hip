// C ABI of the microscaled 4-bit operators (declared in include/bcpnn.h): argument checks, launches
// and the 4-bit layer's ownership.
#include <stdint.h>

#include <algorithm>
#include <new>
#include <vector>

#include "bcpnn_internal.h"
#include "mx_format.h"
#include "mx_layer_layout.h"

using bcpnn::ActiveLists;
using bcpnn::ActiveUnits;
using bcpnn::fail;
using bcpnn::Geometry;

struct bcpnn_mx {
    bcpnn_config cfg;
    Geometry g;
    hipStream_t stream;
    uint8_t* codes = nullptr;
    uint8_t* scales = nullptr;
    float* b = nullptr;
    ActiveUnits act{};
    float* turned = nullptr;             // workspace [n_in][turned_rows]
    int64_t turned_rows = 0;
    bool failed = false;
};

namespace {

constexpr int64_t kMostRows = 1ll << 40;         // of an operand, and columns: byte counts stay in 64 bits
constexpr int64_t kMostWorkgroups = 1ll << 24;   // of 256 work-items: a launch stays below 2^32

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

int element_size(int32_t dtype) {
    return dtype == BCPNN_F32 ? 4 : dtype == BCPNN_F16 || dtype == BCPNN_BF16 ? 2 : 0;
}

bool sizes_ok(int64_t rows, int64_t cols) {
    return rows >= 0 && cols >= 0 && rows <= kMostRows && cols <= kMostRows &&
           bcpnn::mx_row_blocks(rows) <= (1ll << 46) / std::max<int64_t>(1, bcpnn::mx_groups(cols));
}

bcpnn_status check_matrix(const char* what, const void* p, int32_t dtype, int64_t rows, int64_t cols, int64_t ld) {
    const int size = element_size(dtype);
    if (!size) return fail(BCPNN_EINVAL, "unknown element type %d", dtype);
    if (!sizes_ok(rows, cols)) return fail(BCPNN_EINVAL, "matrix sizes out of range");
    if (rows > 1 && ld < cols) return fail(BCPNN_EINVAL, "the row stride of %s is shorter than a row", what);
    if (ld > kMostRows || ld < 0) return fail(BCPNN_EINVAL, "the row stride of %s is out of range", what);
    if (rows && cols && !p) return fail(BCPNN_EINVAL, "%s is required", what);
    if ((uintptr_t)p % size) return fail(BCPNN_EINVAL, "%s is not aligned to its elements", what);
    return BCPNN_OK;
}

bcpnn_status launched(hipError_t e, const char* what) {
    return e == hipSuccess ? BCPNN_OK : fail(BCPNN_EDEVICE, "%s failed: %s", what, hipGetErrorString(e));
}

bcpnn_status making(hipError_t e) {
    return e == hipErrorOutOfMemory ? fail(BCPNN_ENOMEM, "device allocation failed: %s", hipGetErrorString(e))
                                    : launched(e, "making the 4-bit layer");
}

void free_mx(bcpnn_mx* m) {
    if (!m) return;
    void* bufs[] = {m->codes, m->scales, m->b, m->act.units, m->act.count, m->turned};
    for (void* p : bufs)
        if (p) (void)hipFree(p);
    delete m;
}

bcpnn_status usable(const bcpnn_mx* m) {
    if (!m) return fail(BCPNN_EINVAL, "the 4-bit layer is NULL");
    if (m->failed) return fail(BCPNN_ESTATE, "the 4-bit layer failed earlier");
    return BCPNN_OK;
}

bcpnn_status forward(bcpnn_mx* m, const float* x, int32_t B, float* y, float* s, int32_t* winner) {
    const hipError_t e = bcpnn::launch_mx_forward(m->stream, m->g, x, B, m->codes, m->scales, m->b, m->act,
                                                  m->cfg.gain, m->turned, m->turned_rows, y, s, winner);
    if (e != hipSuccess) m->failed = true;
    return launched(e, "the 4-bit forward pass");
}

bcpnn_status check_batch(const bcpnn_mx* m, int32_t B) {
    if (B < 1 || B > m->cfg.max_batch)
        return fail(BCPNN_EINVAL, "batch %d outside [1, %d]", B, m->cfg.max_batch);
    return BCPNN_OK;
}

}  // namespace

namespace bcpnn {

bcpnn_status mx_layer_make(const bcpnn_config& cfg, const float* w, const float* b, const ActiveLists& act,
                           hipStream_t stream, bcpnn_mx** out) {
    bcpnn_mx* m = new (std::nothrow) bcpnn_mx();
    if (!m) return fail(BCPNN_ENOMEM, "out of host memory");
    m->cfg = cfg;
    m->g = Geometry{cfg.in_hcu, cfg.in_mcu, cfg.out_hcu, cfg.out_mcu, (int64_t)cfg.in_hcu * cfg.in_mcu,
                    (int64_t)cfg.out_hcu * cfg.out_mcu};
    m->stream = stream;
    m->turned_rows = mx_forward_turned_rows(m->g, cfg.max_batch);
    m->act.most = act.most * cfg.in_mcu;
    m->act.kg = (int32_t)mx_groups(m->act.most);
    const int64_t blocks = cfg.out_hcu * mx_row_blocks(cfg.out_mcu) * (int64_t)m->act.kg;
    if (blocks >= kMostWorkgroups) {
        free_mx(m);
        return fail(BCPNN_EINVAL, "too many blocks of active weights for one launch");
    }
    const size_t units = (size_t)cfg.out_hcu * m->act.kg * kMxGroup;
    hipError_t e = hipMalloc((void**)&m->codes, blocks * kMxGroupCodes);
    if (e == hipSuccess) e = hipMalloc((void**)&m->scales, blocks * kMxGroupScales);
    if (e == hipSuccess) e = hipMalloc((void**)&m->b, m->g.n_out * sizeof(float));
    if (e == hipSuccess) e = hipMalloc((void**)&m->act.units, units * sizeof(int32_t));
    if (e == hipSuccess) e = hipMalloc((void**)&m->act.count, cfg.out_hcu * sizeof(int32_t));
    if (e == hipSuccess && m->turned_rows)
        e = hipMalloc((void**)&m->turned, m->turned_rows * m->g.n_in * sizeof(float));
    if (e == hipSuccess)
        e = hipMemcpyAsync(m->b, b, m->g.n_out * sizeof(float), hipMemcpyDeviceToDevice, stream);
    if (e == hipSuccess) e = launch_mx_units(stream, m->g, act, m->act);
    if (e == hipSuccess) e = launch_mx_pack(stream, m->g, w, m->act, m->codes, m->scales);
    if (e == hipSuccess) e = mx_forward_prepare();
    const hipError_t waited = hipStreamSynchronize(stream);
    if (e == hipSuccess) e = waited;
    if (e != hipSuccess) {
        free_mx(m);
        return making(e);
    }
    *out = m;
    return BCPNN_OK;
}

}  // namespace bcpnn

extern "C" {

int64_t bcpnn_mx_bytes(int64_t rows, int64_t cols) {
    if (!sizes_ok(rows, cols)) return -1;
    return bcpnn::mx_row_blocks(rows) * bcpnn::mx_groups(cols) * (bcpnn::kMxGroupCodes + bcpnn::kMxGroupScales);
}

bcpnn_status bcpnn_mx_quantize(const void* src_dev, int32_t dtype, int64_t rows, int64_t cols, int64_t ld,
                               void* by_row_dev, void* by_col_dev, void* hip_stream) {
    if (bcpnn_status st = check_matrix("src_dev", src_dev, dtype, rows, cols, ld)) return st;
    if (rows == 0 || cols == 0) return BCPNN_OK;
    if (!by_row_dev && !by_col_dev) return fail(BCPNN_EINVAL, "by_row_dev or by_col_dev is required");
    if (misaligned(by_row_dev) || misaligned(by_col_dev))
        return fail(BCPNN_EINVAL, "MX operands must be 16-byte aligned");
    if (bcpnn::mx_quantize_workgroups(rows, cols, by_col_dev != nullptr) >= kMostWorkgroups)
        return fail(BCPNN_EINVAL, "the matrix is too large for one launch");
    return launched(bcpnn::launch_mx_quantize((hipStream_t)hip_stream, src_dev, dtype, rows, cols, ld, by_row_dev,
                                              by_col_dev), "MX quantisation");
}

bcpnn_status bcpnn_mx_dequantize(const void* mx_dev, int64_t rows, int64_t cols, void* dst_dev, int32_t dtype,
                                 int64_t ld, void* hip_stream) {
    if (bcpnn_status st = check_matrix("dst_dev", dst_dev, dtype, rows, cols, ld)) return st;
    if (rows == 0 || cols == 0) return BCPNN_OK;
    if (!mx_dev || misaligned(mx_dev)) return fail(BCPNN_EINVAL, "mx_dev is required, 16-byte aligned");
    if (bcpnn::mx_quantize_workgroups(rows, cols, false) >= kMostWorkgroups)
        return fail(BCPNN_EINVAL, "the matrix is too large for one launch");
    return launched(bcpnn::launch_mx_dequantize((hipStream_t)hip_stream, mx_dev, rows, cols, dst_dev, dtype, ld),
                    "reading an MX operand");
}

int64_t bcpnn_mx_product_bytes(int64_t m, int64_t n, int64_t k) {
    if (!sizes_ok(m, k) || !sizes_ok(n, k) || !sizes_ok(m, n)) return -1;
    return bcpnn::mx_product_work_bytes(m, n, k);
}

bcpnn_status bcpnn_mx_product(const void* a_dev, const void* b_dev, int64_t m, int64_t n, int64_t k, float alpha,
                              float beta, const float* bias_dev, void* c_dev, int32_t dtype, int64_t ld,
                              void* work_dev, void* hip_stream) {
    if (bcpnn_status st = check_matrix("c_dev", c_dev, dtype, m, n, ld)) return st;
    if (!sizes_ok(m, k) || !sizes_ok(n, k)) return fail(BCPNN_EINVAL, "operand sizes out of range");
    if (m == 0 || n == 0) return BCPNN_OK;
    if (k && (!a_dev || !b_dev)) return fail(BCPNN_EINVAL, "a_dev and b_dev are required");
    if (misaligned(a_dev) || misaligned(b_dev)) return fail(BCPNN_EINVAL, "MX operands must be 16-byte aligned");
    if ((uintptr_t)bias_dev % sizeof(float)) return fail(BCPNN_EINVAL, "bias_dev is not aligned to its elements");
    if (bcpnn::mx_product_work_bytes(m, n, k) && (!work_dev || misaligned(work_dev)))
        return fail(BCPNN_EINVAL, "work_dev of bcpnn_mx_product_bytes is required, 16-byte aligned");
    if (bcpnn::mx_product_work_items(m, n, k) >= 256 * kMostWorkgroups)
        return fail(BCPNN_EINVAL, "the product is too large for one launch");
    return launched(bcpnn::launch_mx_product((hipStream_t)hip_stream, a_dev, b_dev, m, n, k, alpha, beta, bias_dev,
                                             c_dev, dtype, ld, work_dev), "the MX product");
}

bcpnn_status bcpnn_mx_create(const bcpnn_config* cfg, const uint8_t* mask_host, const float* w_dev,
                             const float* b_dev, void* hip_stream, bcpnn_mx** out) try {
    if (!out) return fail(BCPNN_EINVAL, "out is NULL");
    *out = nullptr;
    if (const char* why = bcpnn::check_config(cfg)) return fail(BCPNN_EINVAL, "%s", why);
    if (!w_dev || !b_dev) return fail(BCPNN_EINVAL, "w_dev and b_dev are required");
    if (misaligned(w_dev) || misaligned(b_dev))
        return fail(BCPNN_EINVAL, "device buffers must be 16-byte aligned");
    std::vector<int32_t> list, count;
    int32_t most = 0;
    if (const char* why = bcpnn::build_active_lists(*cfg, mask_host, list, count, most))
        return fail(BCPNN_EINVAL, "%s", why);
    const hipStream_t stream = (hipStream_t)hip_stream;
    int32_t* lists = nullptr;                                // [out_hcu][in_hcu], then the counts
    const size_t n = list.size();
    list.insert(list.end(), count.begin(), count.end());
    hipError_t e = hipMalloc((void**)&lists, list.size() * sizeof(int32_t));
    if (e == hipSuccess)
        e = hipMemcpyAsync(lists, list.data(), list.size() * sizeof(int32_t), hipMemcpyHostToDevice, stream);
    const bcpnn_status st = e != hipSuccess ? making(e)
                                            : bcpnn::mx_layer_make(*cfg, w_dev, b_dev,
                                                                   ActiveLists{lists, lists + n, cfg->in_hcu, most},
                                                                   stream, out);
    (void)hipStreamSynchronize(stream);                      // (the copy, whatever came after it)
    (void)hipFree(lists);
    return st;
} catch (const std::bad_alloc&) {
    return fail(BCPNN_ENOMEM, "out of host memory");
}

void bcpnn_mx_destroy(bcpnn_mx* m) {
    if (!m) return;
    (void)hipStreamSynchronize(m->stream);
    free_mx(m);
}

bcpnn_status bcpnn_mx_forward(bcpnn_mx* m, const float* x_dev, int32_t B, float* y_dev, float* s_dev) {
    if (bcpnn_status st = usable(m)) return st;
    if (!x_dev || !y_dev) return fail(BCPNN_EINVAL, "x_dev and y_dev are required");
    if (misaligned(x_dev) || misaligned(y_dev) || misaligned(s_dev))
        return fail(BCPNN_EINVAL, "device buffers must be 16-byte aligned");
    if (bcpnn_status st = check_batch(m, B)) return st;
    return forward(m, x_dev, B, y_dev, s_dev, nullptr);
}

bcpnn_status bcpnn_mx_readout(bcpnn_mx* m, const float* x_dev, int32_t B, int32_t* winner_dev) {
    if (bcpnn_status st = usable(m)) return st;
    if (!x_dev || !winner_dev) return fail(BCPNN_EINVAL, "x_dev and winner_dev are required");
    if (misaligned(x_dev) || misaligned(winner_dev))
        return fail(BCPNN_EINVAL, "device buffers must be 16-byte aligned");
    if (bcpnn_status st = check_batch(m, B)) return st;
    return forward(m, x_dev, B, nullptr, nullptr, winner_dev);
}

bcpnn_status bcpnn_mx_predict(bcpnn_mx* hidden, bcpnn_mx* readout, const float* x_dev, int32_t B, float* y_dev,
                              int32_t rows, int32_t* winner_dev) {
    if (bcpnn_status st = usable(hidden)) return st;
    if (bcpnn_status st = usable(readout)) return st;
    if (!x_dev || !y_dev || !winner_dev) return fail(BCPNN_EINVAL, "x_dev, y_dev and winner_dev are required");
    if (misaligned(x_dev) || misaligned(y_dev)) return fail(BCPNN_EINVAL, "device buffers must be 16-byte aligned");
    if (readout->g.n_in != hidden->g.n_out || readout->g.out_hcu != 1 || readout->stream != hidden->stream)
        return fail(BCPNN_EINVAL, "the readout must have one HCU over the hidden units, on one stream");
    if (B < 1 || rows < 1) return fail(BCPNN_EINVAL, "B and rows must be positive");
    // Rows at a time: whole row blocks where there are so many.  (Any row of an aligned x will do as the first:
    // it is read as many values at a time as divide a row.)
    const int64_t n_in = hidden->g.n_in;
    const int64_t step = rows >= B || rows < bcpnn::kMxRows ? rows : rows / bcpnn::kMxRows * bcpnn::kMxRows;
    for (int64_t k = 0; k < B; k += step) {
        const int32_t n = (int32_t)std::min<int64_t>(step, B - k);
        if (bcpnn_status st = forward(hidden, x_dev + k * n_in, n, y_dev, nullptr, nullptr)) return st;
        if (bcpnn_status st = forward(readout, y_dev, n, nullptr, nullptr, winner_dev + k)) return st;
    }
    return BCPNN_OK;
}

}  // extern "C"
