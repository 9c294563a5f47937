// C ABI of the operators of a model's layer: checks of the arguments, scratch, launches.  See include/helios.h for the
// contract of every entry point.
#include "context.hpp"
#include "layer.hpp"

#include <algorithm>

using namespace helios;

namespace {

constexpr int64_t kMaxCount = (1ll << 31) - 1024;

int bytes_of(int type) { return type == HELIOS_F32 ? 4 : type == HELIOS_E4M3 ? 1 : 2; }
bool is_float(int type) { return type == HELIOS_F32 || type == HELIOS_F16 || type == HELIOS_BF16; }

constexpr int64_t kMaxSpan = 1ll << 57;           // bytes from a matrix's first row to the end of its last: more than can be addressed
// An array of a call, as its checks see it.
struct Matrix {
    const char* name;
    const void* data;
    int64_t rows, cols, ld;
    int bytes;                                    // of an element
    bool written;
    int64_t pitch() const { return ld * bytes; }
    int64_t extent() const { return rows < 1 ? 0 : (rows - 1) * pitch() + cols * bytes; }
};

bool share_memory(const Matrix& a, const Matrix& b) {
    if (!a.data || !b.data || !overlap(a.data, a.extent(), b.data, b.extent())) return false;
    if (a.pitch() != b.pitch() || a.rows < 1 || a.pitch() < 1) return true;
    // side by side in one wider array?
    const int64_t pitch = a.pitch(), wa = a.cols * a.bytes, wb = b.cols * b.bytes;
    const int64_t apart = reinterpret_cast<intptr_t>(b.data) - reinterpret_cast<intptr_t>(a.data), off = (apart % pitch + pitch) % pitch;
    return off < wa || off + wb > pitch;
}
bool same_matrix(const Matrix& a, const Matrix& b) { return a.data == b.data && a.ld == b.ld && a.bytes == b.bytes && a.cols == b.cols; }

// Pointers, widths, alignment, and that what is written is apart from everything else; `twin[i]` (or -1): the array that
// written array i may be the very same as, as a bit mask.
int check(helios_ctx* c, const Matrix* m, int n, const uint32_t* twins) {
    for (int i = 0; i < n; ++i) {
        if (!m[i].data) continue;
        if (reinterpret_cast<uintptr_t>(m[i].data) % m[i].bytes != 0) return fail(c, HELIOS_EINVAL, "%s is not aligned to its elements", m[i].name);
        if (m[i].ld < m[i].cols && (m[i].written || m[i].ld != 0))
            return fail(c, HELIOS_EINVAL, "%s: rows are %lld elements apart, narrower than %lld", m[i].name, (long long)m[i].ld, (long long)m[i].cols);
        if (m[i].ld > kMaxSpan / m[i].bytes / std::max<int64_t>(m[i].rows, 1)) return fail(c, HELIOS_EINVAL, "%s: rows are too far apart", m[i].name);
    }
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j) {
            if (i == j || !m[i].written || (m[j].written && j < i) || !share_memory(m[i], m[j])) continue;
            if (((twins[i] >> j) & 1) && same_matrix(m[i], m[j])) continue;
            return fail(c, HELIOS_EINVAL, "%s shares memory with %s", m[i].name, m[j].name);
        }
    return HELIOS_OK;
}

int check_counts(helios_ctx* c, const char* call, int64_t n_rows, const int64_t* n_rows_dev) {
    if (n_rows < 0 || n_rows >= kMaxCount) return fail(c, HELIOS_EINVAL, "%s: n_rows must be 0 to 2^31 - 1025 (got %lld)", call, (long long)n_rows);
    if (reinterpret_cast<uintptr_t>(n_rows_dev) % 8 != 0) return fail(c, HELIOS_EINVAL, "%s: n_rows_dev is not aligned", call);
    return HELIOS_OK;
}
int check_width(helios_ctx* c, const char* call, const char* what, int64_t width, int64_t most) {
    if (width < 1 || width > most) return fail(c, HELIOS_EINVAL, "%s: %s must be 1 to %lld (got %lld)", call, what, (long long)most, (long long)width);
    return HELIOS_OK;
}
constexpr int64_t kMaxWidth = 1 << 24;            // of a product's rows

// A table of learnt rows, and the types of its rows and of what is looked up.
int check_table(helios_ctx* c, const char* call, int64_t n_table, int table_type, int y_type) {
    if (n_table < 0 || n_table >= kMaxCount) return fail(c, HELIOS_EINVAL, "%s: n_table must be 0 to 2^31 - 1025 (got %lld)", call, (long long)n_table);
    if (!is_float(table_type)) return fail(c, HELIOS_EINVAL, "%s: unknown table_type %d", call, table_type);
    if (!is_float(y_type) || (y_type != table_type && table_type != HELIOS_F32)) return fail(c, HELIOS_EINVAL, "%s: y_type %d does not go with table_type %d", call, y_type, table_type);
    return HELIOS_OK;
}
int check_drop(helios_ctx* c, const char* call, const helios_drop& d, Drop* out) {
    if (!(d.p >= 0.0 && d.p <= 1.0)) return fail(c, HELIOS_EINVAL, "%s: the share of dropped elements must be 0 to 1", call);
    const uint32_t t = static_cast<uint32_t>(d.p * 65536.0 + 0.5);
    *out = Drop{d.seed, d.seed_dev, d.site, t, t < 65536 ? static_cast<float>(65536.0 / (65536.0 - t)) : 0.0f};
    return HELIOS_OK;
}

// Scratch of at least `bytes` bytes (*at), behind a line of counters that are zero between calls.
constexpr size_t kCounterBytes = sizeof(uint32_t) * kLayerCounters;
int scratch(helios_ctx* c, size_t bytes, char** at) {
    bytes += kCounterBytes;
    *at = static_cast<char*>(c->layer_scratch) + kCounterBytes;
    if (bytes <= c->layer_scratch_bytes) return HELIOS_OK;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    HIP_TRY(c, hipStreamIsCapturing(c->stream, &capture));
    if (capture != hipStreamCaptureStatusNone) return fail(c, HELIOS_ESTATE, "the call needs scratch that it cannot allocate in a capture: make it once outside before");
    const size_t needed = bytes;
    bytes = std::max<size_t>({bytes, 2 * c->layer_scratch_bytes, size_t{1} << 20});
    void* p = nullptr;
    if (c->n_layer_outgrown >= kMostOutgrown) return fail(c, HELIOS_ESTATE, "scratch has grown %d times in short steps: create the context anew", kMostOutgrown);
    hipError_t e = hipMalloc(&p, bytes);
    if (e != hipSuccess && needed < bytes) {      // (no room to grow into: what the call needs may still fit)
        (void)hipGetLastError();
        bytes = needed;
        e = hipMalloc(&p, bytes);
    }
    if (e != hipSuccess) {
        (void)hipGetLastError();                  // (not the next launch's)
        return fail(c, HELIOS_EHIP, "scratch of %zu bytes: %s", bytes, hipGetErrorString(e));
    }
    e = hipMemsetAsync(p, 0, kCounterBytes, c->stream);
    if (e != hipSuccess) {
        (void)hipFree(p);
        return fail(c, HELIOS_EHIP, "hipMemsetAsync: %s", hipGetErrorString(e));
    }
    if (c->layer_scratch) c->layer_outgrown[c->n_layer_outgrown++] = c->layer_scratch;
    c->layer_scratch = p;
    c->layer_scratch_bytes = bytes;
    *at = static_cast<char*>(p) + kCounterBytes;
    return HELIOS_OK;
}

#define TRY(expr)                             \
    do {                                      \
        const int rc_ = (expr);               \
        if (rc_ != HELIOS_OK) return rc_;     \
    } while (0)

}  // namespace

extern "C" {

int helios_linear(helios_ctx* c, const helios_linear_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_linear: NULL arguments");
    TRY(check_counts(c, "helios_linear", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_linear", "n_in", a->n_in, kMaxWidth));
    TRY(check_width(c, "helios_linear", "n_out", a->n_out, kMaxWidth));
    if (a->act < HELIOS_ACT_NONE || a->act > HELIOS_ACT_SILU) return fail(c, HELIOS_EINVAL, "helios_linear: unknown activation %d", a->act);
    const bool in_8_bits = a->x_type == HELIOS_E4M3;
    if (!in_8_bits && !is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_linear: unknown x_type %d", a->x_type);
    if (!is_float(a->out_type) || (!in_8_bits && a->out_type != a->x_type && a->out_type != HELIOS_F32))
        return fail(c, HELIOS_EINVAL, "helios_linear: out_type %d does not go with x_type %d", a->out_type, a->x_type);
    if (a->n_rows == 0) return HELIOS_OK;
    if (!a->x || !a->w || !a->y) return fail(c, HELIOS_EINVAL, "helios_linear: NULL pointer");
    if ((a->x_scale != nullptr) != in_8_bits || (a->w_scale != nullptr) != in_8_bits)
        return fail(c, HELIOS_EINVAL, "helios_linear: x_scale and w_scale go with 8-bit operands, and only with them");
    const int xb = bytes_of(a->x_type), ob = bytes_of(a->out_type);
    const Matrix m[] = {{"x", a->x, a->n_rows, a->n_in, a->x_ld, xb, false},
                        {"w", a->w, a->n_out, a->n_in, a->w_ld, xb, false},
                        {"x_scale", a->x_scale, 1, a->n_rows, a->n_rows, 4, false},
                        {"w_scale", a->w_scale, 1, a->n_out, a->n_out, 4, false},
                        {"bias", a->bias, 1, a->n_out, a->n_out, ob, false},
                        {"residual", a->residual, a->n_rows, a->n_out, a->residual_ld, ob, false},
                        {"pre", a->pre, a->n_rows, a->n_out, a->pre_ld, ob, true},
                        {"y", a->y, a->n_rows, a->n_out, a->y_ld, ob, true}};
    const uint32_t twins[8] = {0, 0, 0, 0, 0, 0, 0, 1u << 5};
    TRY(check(c, m, 8, twins));
    DeviceGuard guard(c->device);
    const LinearJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->n_in), static_cast<int32_t>(a->n_out), a->act, a->x_type, a->out_type,
                        a->x, a->x_ld, a->x_scale, a->w, a->w_ld, a->w_scale, a->bias, a->residual, a->residual_ld, a->pre, a->pre_ld, a->y, a->y_ld};
    HIP_TRY(c, launch_linear(c->stream, job));
    return HELIOS_OK;
}

int helios_linear_grad(helios_ctx* c, const helios_linear_grad_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_linear_grad: NULL arguments");
    TRY(check_counts(c, "helios_linear_grad", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_linear_grad", "n_in", a->n_in, kMaxWidth));
    TRY(check_width(c, "helios_linear_grad", "n_out", a->n_out, kMaxWidth));
    if (a->act < HELIOS_ACT_NONE || a->act > HELIOS_ACT_SILU) return fail(c, HELIOS_EINVAL, "helios_linear_grad: unknown activation %d", a->act);
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_linear_grad: x_type %d has no gradient", a->x_type);
    if (a->out_type != a->x_type && a->out_type != HELIOS_F32)
        return fail(c, HELIOS_EINVAL, "helios_linear_grad: out_type %d does not go with x_type %d", a->out_type, a->x_type);
    if (!a->dx && !a->dw && !a->dbias) return HELIOS_OK;
    const bool slope = a->act != HELIOS_ACT_NONE;
    if (a->n_rows > 0 && (!a->dy || (a->dx && !a->w) || (a->dw && !a->x) || (slope && !a->pre)))
        return fail(c, HELIOS_EINVAL, "helios_linear_grad: NULL pointer");
    const int xb = bytes_of(a->x_type), ob = bytes_of(a->out_type);
    const Matrix m[] = {{"x", a->dw ? a->x : nullptr, a->n_rows, a->n_in, a->x_ld, xb, false},
                        {"w", a->dx ? a->w : nullptr, a->n_out, a->n_in, a->w_ld, xb, false},
                        {"dy", a->dy, a->n_rows, a->n_out, a->dy_ld, ob, false},
                        {"pre", slope ? a->pre : nullptr, a->n_rows, a->n_out, a->pre_ld, ob, false},
                        {"dx", a->dx, a->n_rows, a->n_in, a->dx_ld, xb, true},
                        {"dw", a->dw, a->n_out, a->n_in, a->dw_ld, xb, true},
                        {"dbias", a->dbias, 1, a->n_out, a->n_out, ob, true}};
    const uint32_t twins[7] = {0};
    TRY(check(c, m, 7, twins));
    DeviceGuard guard(c->device);
    const LinearGradJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->n_in), static_cast<int32_t>(a->n_out), a->act, a->x_type, a->out_type,
                            a->x, a->x_ld, a->w, a->w_ld, a->dy, a->dy_ld, a->pre, a->pre_ld, a->dx, a->dx_ld, a->dw, a->dw_ld, a->dbias};
    char* at = nullptr;
    TRY(scratch(c, linear_grad_scratch_bytes(job), &at));
    HIP_TRY(c, launch_linear_grad(c->stream, job, at));
    return HELIOS_OK;
}

int helios_rms_norm(helios_ctx* c, const helios_rms_norm_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_rms_norm: NULL arguments");
    TRY(check_counts(c, "helios_rms_norm", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_rms_norm", "width", a->width, HELIOS_NORM_MAX_WIDTH));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_rms_norm: unknown x_type %d", a->x_type);
    const bool to_8_bits = a->y_type == HELIOS_E4M3;
    if (!to_8_bits && a->y_type != a->x_type) return fail(c, HELIOS_EINVAL, "helios_rms_norm: y_type %d does not go with x_type %d", a->y_type, a->x_type);
    if (!(a->eps >= 0.0f)) return fail(c, HELIOS_EINVAL, "helios_rms_norm: eps must not be negative");
    if (a->n_rows == 0) return HELIOS_OK;
    if (!a->x || !a->y) return fail(c, HELIOS_EINVAL, "helios_rms_norm: NULL pointer");
    if ((a->y_scale != nullptr) != to_8_bits) return fail(c, HELIOS_EINVAL, "helios_rms_norm: y_scale goes with an output in 8 bits, and only with it");
    const int xb = bytes_of(a->x_type), yb = bytes_of(a->y_type);
    const Matrix m[] = {{"x", a->x, a->n_rows, a->width, a->x_ld, xb, false},
                        {"residual", a->residual, a->n_rows, a->width, a->residual_ld, xb, false},
                        {"gain", a->gain, 1, a->width, a->width, xb, false},
                        {"total", a->total, a->n_rows, a->width, a->total_ld, xb, true},
                        {"y", a->y, a->n_rows, a->width, a->y_ld, yb, true},
                        {"y_scale", a->y_scale, 1, a->n_rows, a->n_rows, 4, true},
                        {"inv_rms", a->inv_rms, 1, a->n_rows, a->n_rows, 4, true}};
    const uint32_t twins[7] = {0, 0, 0, 3, 3, 0, 0};
    TRY(check(c, m, 7, twins));
    DeviceGuard guard(c->device);
    const NormJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->x_type, a->y_type, true, a->eps, a->x, a->x_ld, a->residual,
                      a->residual_ld, a->gain, a->total, a->total_ld, a->y, a->y_ld, a->y_scale, a->inv_rms};
    HIP_TRY(c, launch_norm(c->stream, job));
    return HELIOS_OK;
}

int helios_rms_norm_grad(helios_ctx* c, const helios_rms_norm_grad_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_rms_norm_grad: NULL arguments");
    TRY(check_counts(c, "helios_rms_norm_grad", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_rms_norm_grad", "width", a->width, HELIOS_NORM_MAX_WIDTH));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_rms_norm_grad: unknown x_type %d", a->x_type);
    if (!(a->eps >= 0.0f)) return fail(c, HELIOS_EINVAL, "helios_rms_norm_grad: eps must not be negative");
    if (a->n_rows > 0 && (!a->total || !a->dy || !a->dx)) return fail(c, HELIOS_EINVAL, "helios_rms_norm_grad: NULL pointer");
    if (a->n_rows == 0 && !a->dgain) return HELIOS_OK;
    const int xb = bytes_of(a->x_type);
    const Matrix m[] = {{"total", a->total, a->n_rows, a->width, a->total_ld, xb, false},
                        {"gain", a->gain, 1, a->width, a->width, xb, false},
                        {"inv_rms", a->inv_rms, 1, a->n_rows, a->n_rows, 4, false},
                        {"dy", a->dy, a->n_rows, a->width, a->dy_ld, xb, false},
                        {"dtotal", a->dtotal, a->n_rows, a->width, a->dtotal_ld, xb, false},
                        {"dx", a->dx, a->n_rows, a->width, a->dx_ld, xb, true},
                        {"dgain", a->dgain, 1, a->width, a->width, xb, true}};
    const uint32_t twins[7] = {0, 0, 0, 0, 0, 1u | 1u << 3 | 1u << 4, 0};
    TRY(check(c, m, 7, twins));
    DeviceGuard guard(c->device);
    const NormGradJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->x_type, a->eps, a->total, a->total_ld, a->gain, a->inv_rms,
                          a->dy, a->dy_ld, a->dtotal, a->dtotal_ld, a->dx, a->dx_ld, a->dgain};
    char* at = nullptr;
    TRY(scratch(c, norm_grad_scratch_bytes(job), &at));
    HIP_TRY(c, launch_norm_grad(c->stream, job, at));
    return HELIOS_OK;
}

int helios_quantize_rows(helios_ctx* c, int64_t n_rows, const int64_t* n_rows_dev, int64_t width, int32_t x_type, const void* x, int64_t x_ld, void* q,
                         int64_t q_ld, float* q_scale) {
    if (!c) return HELIOS_EINVAL;
    TRY(check_counts(c, "helios_quantize_rows", n_rows, n_rows_dev));
    TRY(check_width(c, "helios_quantize_rows", "width", width, HELIOS_NORM_MAX_WIDTH));
    if (!is_float(x_type)) return fail(c, HELIOS_EINVAL, "helios_quantize_rows: unknown x_type %d", x_type);
    if (n_rows == 0) return HELIOS_OK;
    if (!x || !q || !q_scale) return fail(c, HELIOS_EINVAL, "helios_quantize_rows: NULL pointer");
    const Matrix m[] = {{"x", x, n_rows, width, x_ld, bytes_of(x_type), false}, {"q", q, n_rows, width, q_ld, 1, true}, {"q_scale", q_scale, 1, n_rows, n_rows, 4, true}};
    const uint32_t twins[3] = {0};
    TRY(check(c, m, 3, twins));
    DeviceGuard guard(c->device);
    const NormJob job{Count{n_rows_dev, n_rows}, static_cast<int32_t>(width), x_type, HELIOS_E4M3, false, 0.0f, x, x_ld, nullptr, 0, nullptr, nullptr, 0, q, q_ld, q_scale, nullptr};
    HIP_TRY(c, launch_norm(c->stream, job));
    return HELIOS_OK;
}

int helios_block_mean(helios_ctx* c, const helios_block_mean_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_block_mean: NULL arguments");
    TRY(check_counts(c, "helios_block_mean", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_block_mean", "width", a->width, kMaxWidth));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_block_mean: unknown x_type %d", a->x_type);
    if (a->n_src < 0 || a->n_src >= kMaxCount || a->n_col < 0 || a->n_col >= kMaxCount) return fail(c, HELIOS_EINVAL, "helios_block_mean: n_src and n_col must be 0 to 2^31 - 1025");
    if (a->n_rows == 0) return HELIOS_OK;
    if ((!a->x && a->n_src > 0) || !a->indptr || (!a->col && a->n_col > 0) || !a->mean) return fail(c, HELIOS_EINVAL, "helios_block_mean: NULL pointer");
    const int xb = bytes_of(a->x_type);
    const Matrix m[] = {{"x", a->x, a->n_src, a->width, a->x_ld, xb, false},
                        {"indptr", a->indptr, 1, a->n_rows + 1, a->n_rows + 1, 8, false},
                        {"col", a->col, 1, a->n_col, a->n_col, 4, false},
                        {"row", a->row, 1, a->n_rows, a->n_rows, 4, false},
                        {"mean", a->mean, a->n_rows, a->width, a->mean_ld, xb, true},
                        {"own", a->own, a->n_rows, a->width, a->own_ld, xb, true}};
    const uint32_t twins[6] = {0};
    TRY(check(c, m, 6, twins));
    DeviceGuard guard(c->device);
    const MeanJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->x_type, a->x, a->x_ld, a->n_src, a->indptr, a->col, a->n_col, a->row,
                      a->mean, a->mean_ld, a->own, a->own_ld, c->err};
    HIP_TRY(c, launch_block_mean(c->stream, job));
    return HELIOS_OK;
}

int helios_block_transpose(helios_ctx* c, int64_t n_rows, const int64_t* n_rows_dev, const int64_t* indptr, const int32_t* col, int64_t n_col,
                           const int32_t* row, int64_t n_src, int32_t* src_indptr, int32_t* src_entry) {
    if (!c) return HELIOS_EINVAL;
    TRY(check_counts(c, "helios_block_transpose", n_rows, n_rows_dev));
    if (n_src < 0 || n_src >= kMaxCount || n_col < 0 || n_col >= kMaxCount || n_col + (row ? n_rows : 0) >= kMaxCount)
        return fail(c, HELIOS_EINVAL, "helios_block_transpose: n_src and the entries must be 0 to 2^31 - 1025");
    if (!src_indptr || (n_rows > 0 && !indptr) || (n_col > 0 && (!col || !src_entry)) || (row && n_rows > 0 && !src_entry))
        return fail(c, HELIOS_EINVAL, "helios_block_transpose: NULL pointer");
    const int64_t entries = n_col + (row ? n_rows : 0);
    const Matrix m[] = {{"indptr", indptr, 1, n_rows + 1, n_rows + 1, 8, false},
                        {"col", col, 1, n_col, n_col, 4, false},
                        {"row", row, 1, n_rows, n_rows, 4, false},
                        {"src_indptr", src_indptr, 1, n_src + 1, n_src + 1, 4, true},
                        {"src_entry", src_entry, 1, entries, entries, 4, true}};
    const uint32_t twins[5] = {0};
    TRY(check(c, m, 5, twins));
    DeviceGuard guard(c->device);
    const TransposeJob job{Count{n_rows_dev, n_rows}, indptr, col, n_col, row, n_src, src_indptr, src_entry, c->err};
    char* at = nullptr;
    TRY(scratch(c, block_transpose_scratch_bytes(job), &at));
    HIP_TRY(c, launch_block_transpose(c->stream, job, at));
    return HELIOS_OK;
}

int helios_block_mean_grad(helios_ctx* c, const helios_block_mean_grad_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_block_mean_grad: NULL arguments");
    TRY(check_counts(c, "helios_block_mean_grad", a->n_rows, nullptr));
    TRY(check_width(c, "helios_block_mean_grad", "width", a->width, kMaxWidth));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_block_mean_grad: unknown x_type %d", a->x_type);
    if (a->n_src < 0 || a->n_src >= kMaxCount || a->n_entries < 0 || a->n_entries >= kMaxCount)
        return fail(c, HELIOS_EINVAL, "helios_block_mean_grad: n_src and n_entries must be 0 to 2^31 - 1025");
    if (a->n_src == 0) return HELIOS_OK;
    if (!a->src_indptr || !a->dx || (a->n_entries > 0 && !a->src_entry) || (a->n_rows > 0 && (!a->indptr || !a->dmean)))
        return fail(c, HELIOS_EINVAL, "helios_block_mean_grad: NULL pointer");
    const int xb = bytes_of(a->x_type);
    const Matrix m[] = {{"indptr", a->indptr, 1, a->n_rows + 1, a->n_rows + 1, 8, false},
                        {"src_indptr", a->src_indptr, 1, a->n_src + 1, a->n_src + 1, 4, false},
                        {"src_entry", a->src_entry, 1, a->n_entries, a->n_entries, 4, false},
                        {"dmean", a->dmean, a->n_rows, a->width, a->dmean_ld, xb, false},
                        {"down", a->down, a->n_rows, a->width, a->down_ld, xb, false},
                        {"dx", a->dx, a->n_src, a->width, a->dx_ld, xb, true}};
    const uint32_t twins[6] = {0};
    TRY(check(c, m, 6, twins));
    DeviceGuard guard(c->device);
    const MeanGradJob job{a->n_rows, a->n_src, a->n_entries, static_cast<int32_t>(a->width), a->x_type, a->indptr, a->src_indptr, a->src_entry, a->dmean,
                          a->dmean_ld, a->down, a->down_ld, a->dx, a->dx_ld, c->err};
    char* at = nullptr;
    TRY(scratch(c, block_mean_grad_scratch_bytes(job), &at));
    HIP_TRY(c, launch_block_mean_grad(c->stream, job, reinterpret_cast<uint32_t*>(at - kCounterBytes), at));
    return HELIOS_OK;
}

int helios_embedding(helios_ctx* c, const helios_embedding_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_embedding: NULL arguments");
    TRY(check_counts(c, "helios_embedding", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_embedding", "width", a->width, kMaxWidth));
    TRY(check_table(c, "helios_embedding", a->n_table, a->table_type, a->y_type));
    if (a->n_rows == 0) return HELIOS_OK;
    if (!a->ids || !a->y || (a->n_table > 0 && !a->table)) return fail(c, HELIOS_EINVAL, "helios_embedding: NULL pointer");
    const int tb = bytes_of(a->table_type), yb = bytes_of(a->y_type);
    const Matrix m[] = {{"table", a->table, a->n_table, a->width, a->table_ld, tb, false},
                        {"ids", a->ids, 1, a->n_rows, a->n_rows, 4, false},
                        {"add", a->add, a->n_rows, a->width, a->add_ld, yb, false},
                        {"y", a->y, a->n_rows, a->width, a->y_ld, yb, true}};
    const uint32_t twins[4] = {0, 0, 0, 1u << 2};
    TRY(check(c, m, 4, twins));
    DeviceGuard guard(c->device);
    const EmbeddingJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->table_type, a->y_type, a->scale, a->n_table, a->table,
                           a->table_ld, a->ids, a->add, a->add_ld, a->y, a->y_ld, c->err};
    HIP_TRY(c, launch_embedding(c->stream, job));
    return HELIOS_OK;
}

int helios_embedding_grad(helios_ctx* c, const helios_embedding_grad_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_embedding_grad: NULL arguments");
    TRY(check_counts(c, "helios_embedding_grad", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_embedding_grad", "width", a->width, kMaxWidth));
    TRY(check_table(c, "helios_embedding_grad", a->n_table, a->table_type, a->y_type));
    const bool by_row = !a->dtable && (a->n_table > 0 || a->n_distinct);              // (a table without rows may lie anywhere)
    const int64_t n_out = by_row ? std::min(a->n_rows, a->n_table) : a->n_table;
    if (!by_row && (a->drow || a->row_id || a->n_distinct))
        return fail(c, HELIOS_EINVAL, "helios_embedding_grad: dtable, or drow with row_id and n_distinct, but not both");
    if ((by_row && (!a->n_distinct || (n_out > 0 && (!a->drow || !a->row_id)))) || (a->n_rows > 0 && (!a->ids || !a->dy)))
        return fail(c, HELIOS_EINVAL, "helios_embedding_grad: NULL pointer");
    const int tb = bytes_of(a->table_type), yb = bytes_of(a->y_type);
    const Matrix m[] = {{"ids", a->ids, 1, a->n_rows, a->n_rows, 4, false},
                        {"dy", a->dy, a->n_rows, a->width, a->dy_ld, yb, false},
                        {"dtable", a->dtable, n_out, a->width, a->dtable_ld, tb, true},
                        {"drow", a->drow, n_out, a->width, a->drow_ld, tb, true},
                        {"row_id", a->row_id, 1, n_out, n_out, 4, true},
                        {"n_distinct", a->n_distinct, 1, 1, 1, 8, true}};
    const uint32_t twins[6] = {0};
    TRY(check(c, m, 6, twins));
    if (!by_row && n_out == 0) return HELIOS_OK;
    DeviceGuard guard(c->device);
    const EmbeddingGradJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->table_type, a->y_type, a->scale, a->n_table, a->ids, a->dy,
                               a->dy_ld, by_row ? a->drow : a->dtable, by_row ? a->drow_ld : a->dtable_ld, a->row_id, a->n_distinct, c->err};
    char* at = nullptr;
    TRY(scratch(c, embedding_grad_scratch_bytes(job), &at));
    HIP_TRY(c, launch_embedding_grad(c->stream, job, at));
    return HELIOS_OK;
}

int helios_dropout(helios_ctx* c, const helios_dropout_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_dropout: NULL arguments");
    TRY(check_counts(c, "helios_dropout", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_dropout", "width", a->width, kMaxWidth));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_dropout: unknown x_type %d", a->x_type);
    Drop drop;
    TRY(check_drop(c, "helios_dropout", a->drop, &drop));
    if (a->n_rows == 0) return HELIOS_OK;
    if (!a->x || !a->y) return fail(c, HELIOS_EINVAL, "helios_dropout: NULL pointer");
    const int xb = bytes_of(a->x_type);
    const Matrix m[] = {{"x", a->x, a->n_rows, a->width, a->x_ld, xb, false},
                        {"y", a->y, a->n_rows, a->width, a->y_ld, xb, true},
                        {"seed_dev", a->drop.seed_dev, 1, 1, 1, 8, false}};
    const uint32_t twins[3] = {0, 1u << 0, 0};
    TRY(check(c, m, 3, twins));
    DeviceGuard guard(c->device);
    HIP_TRY(c, launch_dropout(c->stream, DropoutJob{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->x_type, drop, a->x, a->x_ld, a->y, a->y_ld}));
    return HELIOS_OK;
}

int helios_join_norm(helios_ctx* c, const helios_join_norm_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_join_norm: NULL arguments");
    TRY(check_counts(c, "helios_join_norm", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_join_norm", "width", a->width, HELIOS_NORM_MAX_WIDTH));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_join_norm: unknown x_type %d", a->x_type);
    const bool to_8_bits = a->y && a->y_type == HELIOS_E4M3;
    if (a->y && !to_8_bits && a->y_type != a->x_type) return fail(c, HELIOS_EINVAL, "helios_join_norm: y_type %d does not go with x_type %d", a->y_type, a->x_type);
    if (!(a->eps >= 0.0f)) return fail(c, HELIOS_EINVAL, "helios_join_norm: eps must not be negative");
    Drop drop;
    TRY(check_drop(c, "helios_join_norm", a->drop, &drop));
    if (!a->norm_x && (a->gain_x || a->inv_rms_x)) return fail(c, HELIOS_EINVAL, "helios_join_norm: gain_x and inv_rms_x go with a norm of x (norm_x)");
    if (a->n_rows == 0) return HELIOS_OK;
    if (!a->x || (!a->total && !a->y)) return fail(c, HELIOS_EINVAL, "helios_join_norm: NULL pointer");
    if (!a->y && (a->gain || a->inv_rms)) return fail(c, HELIOS_EINVAL, "helios_join_norm: gain and inv_rms go with y");
    if ((a->y_scale != nullptr) != to_8_bits) return fail(c, HELIOS_EINVAL, "helios_join_norm: y_scale goes with an output in 8 bits, and only with it");
    const int xb = bytes_of(a->x_type), yb = bytes_of(a->y ? a->y_type : a->x_type);
    const int64_t gate_ld = a->gate ? a->gate_ld : 0;
    const Matrix m[] = {{"x", a->x, a->n_rows, a->width, a->x_ld, xb, false},
                        {"residual", a->residual, a->n_rows, a->width, a->residual_ld, xb, false},
                        {"total", a->total, a->n_rows, a->width, a->total_ld, xb, true},
                        {"y", a->y, a->n_rows, a->width, a->y_ld, yb, true},
                        {"gain_x", a->gain_x, 1, a->width, a->width, xb, false},
                        {"gate", a->gate, gate_ld ? a->n_rows : 1, a->width, gate_ld ? gate_ld : a->width, xb, false},
                        {"gain", a->gain, 1, a->width, a->width, xb, false},
                        {"y_scale", a->y_scale, 1, a->n_rows, a->n_rows, 4, true},
                        {"inv_rms_x", a->inv_rms_x, 1, a->n_rows, a->n_rows, 4, true},
                        {"inv_rms", a->inv_rms, 1, a->n_rows, a->n_rows, 4, true},
                        {"seed_dev", a->drop.seed_dev, 1, 1, 1, 8, false}};
    const uint32_t twins[11] = {0, 0, 3, 3, 0, 0, 0, 0, 0, 0, 0};
    TRY(check(c, m, 11, twins));
    DeviceGuard guard(c->device);
    const JoinJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->x_type, a->norm_x != 0, a->eps, a->residual_scale, drop, a->x, a->x_ld,
                      a->gain_x, a->gate, gate_ld, a->residual, a->residual_ld, a->gain, a->total, a->total_ld, a->y, a->y_ld, a->y_scale, a->inv_rms_x, a->inv_rms};
    HIP_TRY(c, launch_join(c->stream, job));
    return HELIOS_OK;
}

int helios_join_norm_grad(helios_ctx* c, const helios_join_norm_grad_args* a) {
    if (!c) return HELIOS_EINVAL;
    if (!a) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: NULL arguments");
    TRY(check_counts(c, "helios_join_norm_grad", a->n_rows, a->n_rows_dev));
    TRY(check_width(c, "helios_join_norm_grad", "width", a->width, HELIOS_NORM_MAX_WIDTH));
    if (!is_float(a->x_type)) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: unknown x_type %d", a->x_type);
    if (!(a->eps >= 0.0f)) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: eps must not be negative");
    Drop drop;
    TRY(check_drop(c, "helios_join_norm_grad", a->drop, &drop));
    if (!a->norm_x && (a->gain_x || a->inv_rms_x || a->dgain_x)) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: gain_x, inv_rms_x and dgain_x go with a norm of x (norm_x)");
    if (a->n_rows > 0 && (!a->x || !a->dx || (!a->dy && !a->dtotal) || (a->dy && !a->total))) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: NULL pointer");
    if (a->n_rows > 0 && !a->dy && (a->gain || a->inv_rms || a->dgain)) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: gain, inv_rms and dgain go with dy");
    if (a->dgate && !a->gate && a->n_rows > 0) return fail(c, HELIOS_EINVAL, "helios_join_norm_grad: dgate goes with a gate");
    const int64_t gate_ld = a->gate ? a->gate_ld : 0;
    const bool one_gate = a->gate_ld == 0;
    if (a->n_rows == 0 && !a->dgain && !a->dgain_x && !(a->dgate && one_gate)) return HELIOS_OK;
    const int xb = bytes_of(a->x_type);
    const Matrix m[] = {{"x", a->x, a->n_rows, a->width, a->x_ld, xb, false},
                        {"dy", a->dy, a->n_rows, a->width, a->dy_ld, xb, false},
                        {"total", a->dy ? a->total : nullptr, a->n_rows, a->width, a->total_ld, xb, false},
                        {"dtotal", a->dtotal, a->n_rows, a->width, a->dtotal_ld, xb, false},
                        {"dx", a->dx, a->n_rows, a->width, a->dx_ld, xb, true},
                        {"dresidual", a->dresidual, a->n_rows, a->width, a->dresidual_ld, xb, true},
                        {"dgate", a->dgate, one_gate ? 1 : a->n_rows, a->width, one_gate ? a->width : a->dgate_ld, xb, true},
                        {"dgain_x", a->dgain_x, 1, a->width, a->width, xb, true},
                        {"dgain", a->dgain, 1, a->width, a->width, xb, true},
                        {"gain_x", a->gain_x, 1, a->width, a->width, xb, false},
                        {"gate", a->gate, gate_ld ? a->n_rows : 1, a->width, gate_ld ? gate_ld : a->width, xb, false},
                        {"gain", a->gain, 1, a->width, a->width, xb, false},
                        {"inv_rms_x", a->inv_rms_x, 1, a->n_rows, a->n_rows, 4, false},
                        {"inv_rms", a->inv_rms, 1, a->n_rows, a->n_rows, 4, false},
                        {"seed_dev", a->drop.seed_dev, 1, 1, 1, 8, false}};
    const uint32_t twins[15] = {0, 0, 0, 0, 15u, 14u, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    TRY(check(c, m, 15, twins));
    DeviceGuard guard(c->device);
    const JoinGradJob job{Count{a->n_rows_dev, a->n_rows}, static_cast<int32_t>(a->width), a->x_type, a->norm_x != 0, a->eps, a->residual_scale, drop, a->x, a->x_ld,
                          a->gain_x, a->gate, gate_ld, a->gain, a->total, a->total_ld, a->dy, a->dy_ld, a->dtotal, a->dtotal_ld, a->inv_rms_x, a->inv_rms, a->dx,
                          a->dx_ld, a->dresidual, a->dresidual_ld, one_gate || gate_ld ? a->dgate : nullptr, a->dgate_ld, a->dgain_x, a->dgain};
    char* at = nullptr;
    const size_t bytes = join_grad_scratch_bytes(job);
    if (bytes > 0) TRY(scratch(c, bytes, &at));
    HIP_TRY(c, launch_join_grad(c->stream, job, at));
    return HELIOS_OK;
}

}  // extern "C"
