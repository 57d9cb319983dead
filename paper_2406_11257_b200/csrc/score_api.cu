// The C ABI of the operators that score a restored checkpoint (include/excp.h): argument checks, workspace,
// launches.  No arithmetic lives here.
#include <cmath>

#include "excp_handle.cuh"
#include "score.cuh"

using namespace excp;

namespace excp {
void score_release(ScoreWorkspace& w) {
    if (w.words) cudaFree(w.words);
    if (w.h_flag) cudaFreeHost(w.h_flag);
    w = ScoreWorkspace{};
}
}  // namespace excp

namespace {

constexpr int SCORE_TOP_MAX = 64;

// The workspace, allocated once and cleared on the stream of the call that needs it first.  That call waits for the clearing, so
// that calls on other streams, which nothing orders behind this one, find it done.
bool ensure_score(excp_handle h, cudaStream_t stream) {
    ScoreWorkspace& w = h->score;
    if (w.d_flag) return true;
    if (!w.words) {
        u32* words = nullptr;
        if (!check(h, cudaMalloc(reinterpret_cast<void**>(&words), 64))) return false;
        if (!check(h, cudaMemsetAsync(words, 0, 64, stream)) || !check(h, cudaStreamSynchronize(stream))) {
            cudaFree(words);
            return false;
        }
        w.words = words;
    }
    bool ok = true;
    if (!w.h_flag) {
        ok = check(h, cudaHostAlloc(reinterpret_cast<void**>(&w.h_flag), 64, cudaHostAllocMapped));
        if (ok) *w.h_flag = 0;
    }
    return ok && check(h, cudaHostGetDevicePointer(reinterpret_cast<void**>(&w.d_flag), w.h_flag, 0));   // last: marks it as ready
}

bool dtype_ok(int d) { return d == DT_F32 || d == DT_F16 || d == DT_BF16; }
bool format_ok(int f) { return f == MX4_E8M0_32 || f == MX4_E4M3_16; }
size_t elem_bytes(int d) { return d == DT_F32 ? 4 : 2; }
bool on_element(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype)) == 0; }
bool on_float(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// A matrix in ordinary layout: known type, aligned to its elements, rows that do not overlap.
bool rows_ok(const void* p, int dtype, size_t rows, size_t cols, size_t stride) {
    if (!dtype_ok(dtype) || rows > MX4_MAX_DIM || cols > MX4_MAX_DIM || stride > (1ull << 40)) return false;
    if (rows == 0 || cols == 0) return true;
    return p && on_element(p, dtype) && (rows == 1 || stride >= cols);
}
bool packed_ok(const void* p, size_t rows, size_t cols, int format) {
    if (!format_ok(format) || rows > MX4_MAX_DIM || cols > MX4_MAX_DIM) return false;
    // one launch covers the matrix: its 4-row groups of tiles are counted in 32 bits
    if ((u64)mx4_row_tiles(rows) * mx4_col_tiles(cols) > (1ull << 28)) return false;
    return rows == 0 || cols == 0 || (p && aligned16(p));
}

excp_status finish(excp_handle h) {
    if (!check(h, cudaGetLastError())) return EXCP_ERR_CUDA;
    return EXCP_OK;
}

excp_status matmul_impl(excp_handle h, const void* a, size_t a_rows, const float* a_scale, const void* b, size_t b_rows,
                        const float* b_scale, size_t cols, int format, const float* bias, void* y, int y_dtype,
                        size_t y_stride, cudaStream_t stream, bool behind) {
    const Mx4Operand ma{static_cast<const unsigned char*>(a), a_rows, format == MX4_E4M3_16 ? a_scale : nullptr};
    const Mx4Operand mb{static_cast<const unsigned char*>(b), b_rows, format == MX4_E4M3_16 ? b_scale : nullptr};
    const Mx4Result r{y, y_dtype, y_stride, bias};
    if (!launch_mx4_matmul(h->sms, stream, ma, mb, cols, format, r, h->wait_limit_ns, h->score.d_flag, behind)) {
        check(h, cudaGetLastError());
        return EXCP_ERR_CUDA;
    }
    return finish(h);
}

bool product_ok(size_t a_rows, size_t b_rows, const float* a_scale, const float* b_scale, const float* bias, const void* y,
                int y_dtype, size_t y_stride) {
    if (!rows_ok(y, y_dtype, a_rows, b_rows, y_stride)) return false;
    // tiles of the result are counted in 32 bits
    if ((u64)mx4_row_tiles(a_rows) * mx4_row_tiles(b_rows) > (1ull << 30)) return false;
    return on_float(a_scale) && on_float(b_scale) && on_float(bias);
}

}  // namespace

extern "C" {

size_t excp_mx4_bytes(size_t rows, size_t cols, int format) {
    if (!format_ok(format) || rows > MX4_MAX_DIM || cols > MX4_MAX_DIM) return 0;
    return (size_t)mx4_bytes(rows, cols, format);
}

excp_status excp_mx4_tensor_scale(excp_handle h, const void* x, int dtype, size_t rows, size_t cols, size_t row_stride,
                                  float* scale_out, void* cuda_stream) {
    if (!h || !scale_out || !on_float(scale_out) || !rows_ok(x, dtype, rows, cols, row_stride)) return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!guard.ok || !ensure_score(h, stream)) return EXCP_ERR_CUDA;
    launch_mx4_tensor_scale(h->sms, stream, RowsIn{x, dtype, cols ? rows : 0, cols, row_stride}, h->score.words, scale_out);
    return finish(h);
}

excp_status excp_mx4_quantize(excp_handle h, const void* x, int dtype, size_t rows, size_t cols, size_t row_stride,
                              int format, const float* tensor_scale, void* packed_out, void* cuda_stream) {
    if (!h || !rows_ok(x, dtype, rows, cols, row_stride) || !packed_ok(packed_out, rows, cols, format) || !on_float(tensor_scale))
        return EXCP_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return EXCP_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_mx4_quantize(h->sms, static_cast<cudaStream_t>(cuda_stream), RowsIn{x, dtype, rows, cols, row_stride}, format, tensor_scale,
                        static_cast<unsigned char*>(packed_out));
    return finish(h);
}

excp_status excp_mx4_dequantize(excp_handle h, const void* packed, size_t rows, size_t cols, int format,
                                const float* tensor_scale, void* out, int dtype, size_t row_stride, void* cuda_stream) {
    if (!h || !rows_ok(out, dtype, rows, cols, row_stride) || !packed_ok(packed, rows, cols, format) || !on_float(tensor_scale))
        return EXCP_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return EXCP_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_mx4_dequantize(h->sms, static_cast<cudaStream_t>(cuda_stream), static_cast<const unsigned char*>(packed), rows, cols, format,
                          tensor_scale, out, dtype, row_stride);
    return finish(h);
}

excp_status excp_mx4_matmul(excp_handle h, const void* a, size_t a_rows, const float* a_scale, const void* b, size_t b_rows,
                            const float* b_scale, size_t cols, int format, const float* bias, void* y, int y_dtype,
                            size_t y_row_stride, void* cuda_stream) {
    if (!h || !packed_ok(a, a_rows, cols, format) || !packed_ok(b, b_rows, cols, format) ||
        !product_ok(a_rows, b_rows, a_scale, b_scale, bias, y, y_dtype, y_row_stride))
        return EXCP_ERR_INVALID_ARG;
    if (a_rows == 0 || b_rows == 0) return EXCP_OK;
    DeviceGuard guard(h->device);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!guard.ok || !ensure_score(h, stream)) return EXCP_ERR_CUDA;
    return matmul_impl(h, a, a_rows, a_scale, b, b_rows, b_scale, cols, format, bias, y, y_dtype, y_row_stride, stream, false);
}

size_t excp_mx4_linear_scratch(excp_handle h, size_t rows, size_t w_rows, size_t cols, int format) {
    if (!h || !rows || !w_rows || mx4_linear_in_one(h->sms, rows, w_rows, cols)) return 0;
    return excp_mx4_bytes(rows, cols, format);
}

excp_status excp_mx4_linear(excp_handle h, const void* x, int x_dtype, size_t rows, size_t x_row_stride, const float* x_scale,
                            const void* w, size_t w_rows, const float* w_scale, size_t cols, int format, const float* bias,
                            void* y, int y_dtype, size_t y_row_stride, void* x_packed, void* cuda_stream) {
    if (!h || !rows_ok(x, x_dtype, rows, cols, x_row_stride) ||
        !packed_ok(w, w_rows, cols, format) || !product_ok(rows, w_rows, x_scale, w_scale, bias, y, y_dtype, y_row_stride))
        return EXCP_ERR_INVALID_ARG;
    if (rows == 0 || w_rows == 0) return EXCP_OK;
    const bool direct = mx4_linear_in_one(h->sms, rows, w_rows, cols);     // no packed x: x_packed is not looked at
    if (!direct && !packed_ok(x_packed, rows, cols, format)) return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!guard.ok || !ensure_score(h, stream)) return EXCP_ERR_CUDA;
    if (direct) {
        const Mx4Operand mw{static_cast<const unsigned char*>(w), w_rows, format == MX4_E4M3_16 ? w_scale : nullptr};
        if (!launch_mx4_linear(h->sms, stream, RowsIn{x, x_dtype, rows, cols, x_row_stride}, format == MX4_E4M3_16 ? x_scale : nullptr, mw, format,
                               Mx4Result{y, y_dtype, y_row_stride, bias}, h->wait_limit_ns, h->score.d_flag)) {
            check(h, cudaGetLastError());
            return EXCP_ERR_CUDA;
        }
        return finish(h);
    }
    if (cols)
        launch_mx4_quantize(h->sms, stream, RowsIn{x, x_dtype, rows, cols, x_row_stride}, format, x_scale, static_cast<unsigned char*>(x_packed));
    return matmul_impl(h, x_packed, rows, x_scale, w, w_rows, w_scale, cols, format, bias, y, y_dtype, y_row_stride, stream, cols != 0);
}

excp_status excp_token_logprobs(excp_handle h, const void* logits, int dtype, size_t rows, size_t vocab, size_t row_stride,
                                const long long* tokens, float scale, int top, float* logprob_out, float* entropy_out,
                                float* row_stats_out, float* top_logprob_out, long long* top_index_out, void* cuda_stream) {
    if (!h || !rows_ok(logits, dtype, rows, vocab, row_stride) || !(scale > 0.f) || scale > 1e30f) return EXCP_ERR_INVALID_ARG;
    if (top < 0 || top > SCORE_TOP_MAX || (size_t)top > vocab) return EXCP_ERR_INVALID_ARG;
    if (rows == 0) return EXCP_OK;
    if (!tokens || !logprob_out || (reinterpret_cast<uintptr_t>(tokens) & 7u) || !on_float(logprob_out) || !on_float(entropy_out) ||
        !aligned16(row_stats_out))
        return EXCP_ERR_INVALID_ARG;
    if (top && (!top_logprob_out || !top_index_out || !on_float(top_logprob_out) || (reinterpret_cast<uintptr_t>(top_index_out) & 7u)))
        return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_token_logprobs(h->sms, static_cast<cudaStream_t>(cuda_stream), RowsIn{logits, dtype, rows, vocab, row_stride}, tokens, scale,
                          LogprobsOut{logprob_out, entropy_out, row_stats_out, top, top_logprob_out, top_index_out});
    return finish(h);
}

excp_status excp_token_logprobs_grad(excp_handle h, const void* logits, int dtype, size_t rows, size_t vocab, size_t row_stride,
                                     const long long* tokens, float scale, const float* row_stats, const float* g_logprob,
                                     const float* g_entropy, void* grad_out, size_t grad_row_stride, void* cuda_stream) {
    if (!h || !rows_ok(logits, dtype, rows, vocab, row_stride) || !rows_ok(grad_out, dtype, rows, vocab, grad_row_stride) ||
        !(scale > 0.f) || scale > 1e30f)
        return EXCP_ERR_INVALID_ARG;
    if (rows == 0 || vocab == 0) return EXCP_OK;
    if (!tokens || !row_stats || (reinterpret_cast<uintptr_t>(tokens) & 7u) || !aligned16(row_stats) || !on_float(g_logprob) || !on_float(g_entropy))
        return EXCP_ERR_INVALID_ARG;
    if (grad_out == logits && grad_row_stride != row_stride) return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok) return EXCP_ERR_CUDA;
    launch_token_logprobs_grad(h->sms, static_cast<cudaStream_t>(cuda_stream), RowsIn{logits, dtype, rows, vocab, row_stride}, tokens, scale,
                               row_stats, g_logprob, g_entropy, grad_out, grad_row_stride);
    return finish(h);
}

excp_status excp_score_status(excp_handle h, void* cuda_stream) {
    if (!h) return EXCP_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok || !check(h, cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)))) return EXCP_ERR_CUDA;
    if (!h->score.h_flag) return EXCP_OK;
    const u32 flag = *static_cast<volatile u32*>(h->score.h_flag);
    *static_cast<volatile u32*>(h->score.h_flag) = 0;
    return flag ? EXCP_ERR_TIMEOUT : EXCP_OK;
}

}  // extern "C"
