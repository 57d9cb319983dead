// The C ABI of the layers before the logits and the way back through them (include/excp.h): argument checks, launches.  No
// arithmetic lives here.
#include "api_checks.cuh"
#include "product.cuh"

using namespace excp;

namespace {

bool on8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// Absent where it is null.
Matrix matrix(const excp_matrix* m) {
    Matrix r;
    if (!m || !m->data) return r;
    r.p = m->data;
    r.dtype = m->dtype;
    r.rows = m->rows;
    r.cols = m->cols;
    r.stride = m->rows == 1 ? m->cols : m->row_stride;
    return r;
}
bool plain_ok(const excp_matrix* m) { return m && rows_ok(m->data, m->dtype, m->rows, m->cols, m->row_stride); }
bool same_shape(const excp_matrix* a, const excp_matrix* b) { return a->rows == b->rows && a->cols == b->cols; }
bool empty(const excp_matrix* m) { return m->rows == 0 || m->cols == 0; }
// A matrix in ordinary layout or in 8 bits.
bool kept_ok(const excp_matrix* m) {
    if (!m || m->dtype != EXCP_ACT8) return plain_ok(m);
    return m->rows <= MX4_MAX_DIM && m->cols <= MX4_MAX_DIM && (empty(m) || (m->data && aligned16(m->data)));
}
// An optional one like `of`, of type `dtype` (any plain one: -1).
bool optional_ok(const excp_matrix* m, const excp_matrix* of, int dtype) {
    return !m || (plain_ok(m) && same_shape(m, of) && (dtype < 0 || m->dtype == dtype));
}
// A result may take an input's place where that is said, but then value by value.
bool in_place_ok(const excp_matrix* in, const excp_matrix* out) {
    return !in || !out || empty(out) || in->data != out->data || (in->dtype == out->dtype && (out->rows == 1 || in->row_stride == out->row_stride));
}
bool vector_ok(const void* p, int dtype) { return !p || (dtype_ok(dtype) && on_element(p, dtype)); }
bool act_ok(int act) { return act >= ACT_NONE && act <= ACT_SILU; }

// Whether a tensor map can describe it as it is.
bool on16(const Matrix& m) { return (reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && (m.rows == 1 || m.stride % 8 == 0); }
size_t tidy_bytes(const Matrix& m) { return !m.p || !m.rows || !m.cols || on16(m) ? 0 : (size_t)(m.rows * tidy_pitch(m.cols) * 2); }

bool operand_ok(const excp_matrix* m) { return plain_ok(m) && (m->dtype == EXCP_F16 || m->dtype == EXCP_BF16); }

// c = op(a) op(b)^T, the k values along the rows of a (b) or down its columns.
excp_status product(excp_handle h, const excp_matrix* ma, bool a_along_k, const excp_matrix* mb, bool b_along_k, const ProductEnd& end, void* scratch,
                    void* cuda_stream) {
    Matrix a = matrix(ma), b = matrix(mb);
    const size_t need = tidy_bytes(a) + tidy_bytes(b);
    if (need && (!scratch || !aligned16(scratch))) return EXCP_ERR_INVALID_ARG;
    const u64 tiles = ((end.y.rows + 127) / 128) * ((end.y.cols + 127) / 128);
    if (tiles > (1ull << 27)) return EXCP_ERR_INVALID_ARG;      // counted in 32 bits, in up to eight parts
    DeviceGuard guard(h->device);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!guard.ok || !ensure_score(h, stream)) return EXCP_ERR_CUDA;
    unsigned char* room = static_cast<unsigned char*>(scratch);
    for (Matrix* m : {&a, &b}) {
        const size_t bytes = tidy_bytes(*m);
        if (bytes) {
            launch_tidy(h->sms, stream, *m, room);
            m->p = room;
            m->stride = tidy_pitch(m->cols);
            room += bytes;
        }
        if (m->rows == 1) m->stride = tidy_pitch(m->cols);      // not used, but has to be on 16 bytes
    }
    auto operand = [](const Matrix& m, const excp_matrix* shape, bool along_k) {
        return ProductOperand{m.p, along_k ? shape->rows : shape->cols, along_k ? shape->cols : shape->rows, m.stride, along_k};
    };
    const ProductCall c{operand(a, ma, a_along_k), operand(b, mb, b_along_k), end, ma->dtype, h->device, h->sms, h->wait_limit_ns, h->score.d_flag};
    if (!launch_product(stream, c)) {
        check(h, cudaGetLastError());
        return EXCP_ERR_CUDA;
    }
    return finish(h);
}

}  // namespace

extern "C" {

size_t excp_act8_bytes(size_t rows, size_t cols) {
    if (rows > MX4_MAX_DIM || cols > MX4_MAX_DIM) return 0;
    return (size_t)a8_bytes(rows, cols);
}

excp_status excp_act8_quantize(excp_handle h, const excp_matrix* x, void* packed_out, void* cuda_stream) {
    if (!h || !plain_ok(x)) return EXCP_ERR_INVALID_ARG;
    if (empty(x)) return EXCP_OK;
    if (!packed_out || !aligned16(packed_out)) return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_act8_quantize(static_cast<cudaStream_t>(cuda_stream), matrix(x), static_cast<unsigned char*>(packed_out));
    return finish(h);
}

excp_status excp_act8_restore(excp_handle h, const void* packed, const excp_matrix* out, void* cuda_stream) {
    if (!h || !plain_ok(out)) return EXCP_ERR_INVALID_ARG;
    if (empty(out)) return EXCP_OK;
    if (!packed || !aligned16(packed)) return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_act8_restore(static_cast<cudaStream_t>(cuda_stream), static_cast<const unsigned char*>(packed), matrix(out));
    return finish(h);
}

size_t excp_act_grad_scratch(excp_handle h, size_t rows, size_t cols) { return h ? (size_t)act_grad_scratch(h->sms, rows, cols) : 0; }

excp_status excp_act_grad(excp_handle h, int act, const excp_matrix* dy, const excp_matrix* pre, const excp_matrix* dpre_out, const excp_matrix* again_out,
                          float* dbias_out, void* scratch, void* cuda_stream) {
    if (!h || !act_ok(act) || !plain_ok(dy) || !optional_ok(dpre_out, dy, dy->dtype) || !optional_ok(again_out, dy, dy->dtype) || !in_place_ok(dy, dpre_out) || !on_float(dbias_out))
        return EXCP_ERR_INVALID_ARG;
    if (act == ACT_NONE) {
        if (pre || again_out) return EXCP_ERR_INVALID_ARG;
    } else if (!kept_ok(pre) || !same_shape(pre, dy) || (pre->dtype != EXCP_ACT8 && pre->dtype != dy->dtype)) {
        return EXCP_ERR_INVALID_ARG;
    }
    if (dy->cols == 0) return EXCP_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (dy->rows == 0) return !dbias_out || check(h, cudaMemsetAsync(dbias_out, 0, dy->cols * sizeof(float), stream)) ? EXCP_OK : EXCP_ERR_CUDA;
    if (dbias_out && act_grad_scratch(h->sms, dy->rows, dy->cols) && (!scratch || !aligned16(scratch))) return EXCP_ERR_INVALID_ARG;
    launch_act_grad(h->sms, stream, act, matrix(dy), matrix(pre), matrix(dpre_out), matrix(again_out), dbias_out, static_cast<float*>(scratch));
    return finish(h);
}

excp_status excp_layer_norm(excp_handle h, const excp_matrix* x, const void* weight, const void* bias, int vector_dtype, float eps, int rms,
                            const excp_matrix* y_out, float* row_stats_out, void* kept_out, void* cuda_stream) {
    if (!h || !plain_ok(x) || !plain_ok(y_out) || !same_shape(x, y_out) || x->dtype != y_out->dtype || !in_place_ok(x, y_out) || !(eps >= 0.f) || eps > 1e30f ||
        !vector_ok(weight, vector_dtype) || !vector_ok(bias, vector_dtype) || ((weight || bias) && vector_dtype != EXCP_F32 && vector_dtype != x->dtype) ||
        (rms && bias) || !on8(row_stats_out) || !aligned16(kept_out))
        return EXCP_ERR_INVALID_ARG;
    if (empty(x)) return EXCP_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_layer_norm(h->sms, static_cast<cudaStream_t>(cuda_stream), matrix(x), ColumnVector{weight, vector_dtype}, ColumnVector{bias, vector_dtype}, eps, rms != 0,
                      matrix(y_out), row_stats_out, static_cast<unsigned char*>(kept_out));
    return finish(h);
}

size_t excp_layer_norm_grad_scratch(excp_handle h, size_t rows, size_t cols) { return h ? (size_t)layer_norm_grad_scratch(h->sms, rows, cols) : 0; }

excp_status excp_layer_norm_grad(excp_handle h, const excp_matrix* dy, const excp_matrix* x, const void* weight, int vector_dtype, int rms,
                                 const float* row_stats, const excp_matrix* add, const excp_matrix* dx_out, float* dweight_out, float* dbias_out, void* scratch,
                                 void* cuda_stream) {
    if (!h || !plain_ok(dy) || !kept_ok(x) || !same_shape(x, dy) || (x->dtype != EXCP_ACT8 && x->dtype != dy->dtype) || !vector_ok(weight, vector_dtype) ||
        (weight && vector_dtype != EXCP_F32 && vector_dtype != dy->dtype) || !optional_ok(add, dy, dy->dtype) || !optional_ok(dx_out, dy, dy->dtype) ||
        (add && !dx_out) || !in_place_ok(dy, dx_out) || !in_place_ok(add, dx_out) || !on_float(dweight_out) || !on_float(dbias_out) || !on8(row_stats))
        return EXCP_ERR_INVALID_ARG;
    if (dy->cols == 0) return EXCP_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (dy->rows == 0) {
        for (float* p : {dweight_out, dbias_out})
            if (p && !check(h, cudaMemsetAsync(p, 0, dy->cols * sizeof(float), stream))) return EXCP_ERR_CUDA;
        return EXCP_OK;
    }
    if (!row_stats) return EXCP_ERR_INVALID_ARG;
    if (layer_norm_grad_scratch(h->sms, dy->rows, dy->cols) && (!scratch || !aligned16(scratch))) return EXCP_ERR_INVALID_ARG;
    launch_layer_norm_grad(h->sms, stream, matrix(dy), matrix(x), ColumnVector{weight, vector_dtype}, rms != 0, row_stats, matrix(add), matrix(dx_out),
                           dweight_out, dbias_out, static_cast<float*>(scratch));
    return finish(h);
}

size_t excp_linear_scratch(const excp_matrix* a, const excp_matrix* b) {
    return (a && operand_ok(a) ? tidy_bytes(matrix(a)) : 0) + (b && operand_ok(b) ? tidy_bytes(matrix(b)) : 0);
}

excp_status excp_linear(excp_handle h, const excp_matrix* x, const excp_matrix* w, const void* bias, int bias_dtype, int act, const excp_matrix* residual,
                        const excp_matrix* y_out, const excp_matrix* kept_out, void* scratch, void* cuda_stream) {
    if (!h || !operand_ok(x) || !operand_ok(w) || x->dtype != w->dtype || x->cols != w->cols || !plain_ok(y_out) || y_out->rows != x->rows ||
        y_out->cols != w->rows || !vector_ok(bias, bias_dtype) || !act_ok(act) || !optional_ok(residual, y_out, -1) || !in_place_ok(residual, y_out) ||
        (kept_out && (!kept_ok(kept_out) || !same_shape(kept_out, y_out))))
        return EXCP_ERR_INVALID_ARG;
    if (empty(y_out)) return EXCP_OK;
    return product(h, x, true, w, true, ProductEnd{matrix(y_out), ColumnVector{bias, bias_dtype}, act, matrix(residual), matrix(kept_out)}, scratch, cuda_stream);
}

excp_status excp_linear_grad_input(excp_handle h, const excp_matrix* dy, const excp_matrix* w, const excp_matrix* add, const excp_matrix* dx_out, void* scratch,
                                   void* cuda_stream) {
    if (!h || !operand_ok(dy) || !operand_ok(w) || dy->dtype != w->dtype || dy->cols != w->rows || !plain_ok(dx_out) || dx_out->rows != dy->rows ||
        dx_out->cols != w->cols || !optional_ok(add, dx_out, -1) || !in_place_ok(add, dx_out))
        return EXCP_ERR_INVALID_ARG;
    if (empty(dx_out)) return EXCP_OK;
    return product(h, dy, true, w, false, ProductEnd{matrix(dx_out), ColumnVector{}, ACT_NONE, matrix(add), Matrix{}}, scratch, cuda_stream);
}

excp_status excp_linear_grad_weight(excp_handle h, const excp_matrix* dy, const excp_matrix* x, const excp_matrix* add, const excp_matrix* dw_out, void* scratch,
                                    void* cuda_stream) {
    if (!h || !operand_ok(dy) || !operand_ok(x) || dy->dtype != x->dtype || dy->rows != x->rows || !plain_ok(dw_out) || dw_out->rows != dy->cols ||
        dw_out->cols != x->cols || !optional_ok(add, dw_out, -1) || !in_place_ok(add, dw_out))
        return EXCP_ERR_INVALID_ARG;
    if (empty(dw_out)) return EXCP_OK;
    return product(h, dy, false, x, false, ProductEnd{matrix(dw_out), ColumnVector{}, ACT_NONE, matrix(add), Matrix{}}, scratch, cuda_stream);
}

}  // extern "C"
