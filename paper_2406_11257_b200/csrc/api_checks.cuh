// Checks of arguments that the C entry points of the scoring calls and of the layers share.
#pragma once
#include "excp_handle.cuh"
#include "score.cuh"

namespace excp {
// The workspace of the scoring calls (score_api.cu).
bool ensure_score(excp_handle h, cudaStream_t stream);

inline bool dtype_ok(int d) { return d == DT_F32 || d == DT_F16 || d == DT_BF16; }
inline size_t elem_bytes(int d) { return d == DT_F32 ? 4 : 2; }
inline bool on_element(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype)) == 0; }
inline bool on_float(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// A matrix in ordinary layout: known type, aligned to its elements, rows that do not overlap.
inline bool rows_ok(const void* p, int dtype, size_t rows, size_t cols, size_t stride) {
    if (!dtype_ok(dtype) || rows > MX4_MAX_DIM || cols > MX4_MAX_DIM || stride > (1ull << 40)) return false;
    if (rows == 0 || cols == 0) return true;
    return p && on_element(p, dtype) && (rows == 1 || stride >= cols);
}

inline excp_status finish(excp_handle h) {
    if (!check(h, cudaGetLastError())) return EXCP_ERR_CUDA;
    return EXCP_OK;
}
}  // namespace excp
