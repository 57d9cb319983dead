// Operators that score a restored checkpoint: microscaled 4-bit matrices, their product, log probabilities
// of tokens.  Shared declarations: the packed layout, the workspace, the launch wrappers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "excp_common.cuh"

namespace excp {

// Element types of activations, logits and results (excp_dtype; the weight formats' numbers).
enum DType { DT_F32 = 0, DT_F16 = 1, DT_BF16 = 2 };
enum Mx4Format { MX4_E8M0_32 = 1, MX4_E4M3_16 = 2 };

// ---- packed 4-bit matrices (layout: include/excp.h) ---------------------------
constexpr int MX4_ROWS = 128;                     // rows of a tile = rows of one tensor-core operand
constexpr int MX4_COLS = 256;                     // columns of a tile = 128 bytes of codes, one swizzle span
constexpr int MX4_PIECE = 512;                    // scales of 128 rows x 4 blocks, as the tensor core reads them
constexpr u64 MX4_MAX_DIM = 1ull << 30;

__host__ __device__ constexpr int mx4_block(int fmt) { return fmt == MX4_E4M3_16 ? 16 : 32; }
__host__ __device__ constexpr int mx4_pieces(int fmt) { return MX4_COLS / mx4_block(fmt) / 4; }   // per tile
__host__ __device__ constexpr int mx4_scale_bytes(int fmt) { return mx4_pieces(fmt) * MX4_PIECE; }
__host__ __device__ inline u32 mx4_col_tiles(u64 cols) { return (u32)((cols + MX4_COLS - 1) / MX4_COLS); }
__host__ __device__ inline u32 mx4_row_tiles(u64 rows) { return (u32)((rows + MX4_ROWS - 1) / MX4_ROWS); }
// Rows of codes that row tile `rt` holds: 128, or what is left rounded up to 8.
__host__ __device__ inline u32 mx4_tile_height(u64 rows, u32 rt) {
    const u64 left = rows - (u64)rt * MX4_ROWS;
    return left >= MX4_ROWS ? (u32)MX4_ROWS : (u32)((left + 7) & ~7ull);
}
__host__ __device__ inline u64 mx4_tile_offset(u64 rows, u32 col_tiles, int fmt, u32 rt, u32 ct) {
    const u64 s = mx4_scale_bytes(fmt);
    return (u64)rt * col_tiles * (MX4_ROWS * 128 + s) + (u64)ct * (mx4_tile_height(rows, rt) * 128 + s);
}
__host__ __device__ inline u64 mx4_bytes(u64 rows, u64 cols, int fmt) {
    const u64 ct = mx4_col_tiles(cols), rt = mx4_row_tiles(rows);
    return ct * (((rows + 7) & ~7ull) * 128 + rt * mx4_scale_bytes(fmt));
}

// ---- workspace of a handle, allocated by the first call that needs it ----------
struct ScoreWorkspace {
    u32* words = nullptr;            // device: running maximum and arrival count of the tensor scale; zero between calls
    u32* h_flag = nullptr;           // pinned host word, mapped: a bounded wait of the product ran out
    u32* d_flag = nullptr;           // its device address
};
void score_release(ScoreWorkspace& w);

// ---- launch wrappers --------------------------------------------------------------
struct RowsIn {                      // a matrix in ordinary layout: rows of `cols` values, `stride` values apart
    const void* p;
    int dtype;
    u64 rows, cols, stride;
};
void launch_mx4_tensor_scale(int sms, cudaStream_t s, const RowsIn& x, u32* words, float* scale_out);
void launch_mx4_quantize(int sms, cudaStream_t s, const RowsIn& x, int fmt, const float* tensor_scale, unsigned char* out);
void launch_mx4_dequantize(int sms, cudaStream_t s, const unsigned char* packed, u64 rows, u64 cols, int fmt,
                           const float* tensor_scale, void* out, int dtype, u64 stride);

struct Mx4Operand {
    const unsigned char* p;
    u64 rows;
    const float* scale;              // tensor scale, device; null = 1
};
struct Mx4Result {
    void* y;                         // y[a row, b row]
    int dtype;
    u64 stride;
    const float* bias;               // one per row of b, device; null = none
};
// `behind`: the launch before packs a, and nothing but a depends on it.  False if the launch was refused (cudaGetLastError
// then says why).
bool launch_mx4_matmul(int sms, cudaStream_t s, const Mx4Operand& a, const Mx4Operand& b, u64 cols, int fmt,
                       const Mx4Result& r, u64 wait_ns, u32* flag, bool behind);

// x quantised within the product: where mx4_linear_in_one says so (few rows of few columns to a CTA).
bool mx4_linear_in_one(int sms, u64 rows, u64 w_rows, u64 cols);
bool launch_mx4_linear(int sms, cudaStream_t s, const RowsIn& x, const float* x_scale, const Mx4Operand& w, int fmt,
                       const Mx4Result& r, u64 wait_ns, u32* flag);
bool launch_mx4_matmul_wide(int sms, cudaStream_t s, const Mx4Operand& a, const Mx4Operand& b, u64 cols, int fmt,
                            const Mx4Result& r, u64 wait_ns, u32* flag, bool behind);

struct LogprobsOut {
    float* logprob;
    float* entropy;
    float* row_stats;                // 4 per row: largest logit (not scaled), sum of exp, entropy, 0
    int top;
    float* top_logprob;
    long long* top_index;
};
void launch_token_logprobs(int sms, cudaStream_t s, const RowsIn& logits, const long long* tokens, float scale,
                           const LogprobsOut& out);
void launch_token_logprobs_grad(int sms, cudaStream_t s, const RowsIn& logits, const long long* tokens, float scale,
                                const float* row_stats, const float* g_logprob, const float* g_entropy, void* grad,
                                u64 grad_stride);

#ifdef __CUDACC__
template <int DT> struct ElemOf;
template <> struct ElemOf<DT_F32> { typedef float type; };
template <> struct ElemOf<DT_F16> { typedef __half type; };
template <> struct ElemOf<DT_BF16> { typedef __nv_bfloat16 type; };

// Eight consecutive values at p[0..7] as fp32, in 16-byte loads (p on 16 bytes).
__device__ __forceinline__ void load8(const float* p, float v[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float v[8]) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
    const T* h = reinterpret_cast<const T*>(&a);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = wget(h, k);
}

// 16 bytes from byte `shift` (0 .. 15) of the 32 that a and b hold.
__device__ __forceinline__ uint4 cut16(uint4 a, uint4 b, u32 shift) {
    u32 w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (shift & 8) {
#pragma unroll
        for (int k = 0; k < 6; ++k) w[k] = w[k + 2];
    }
    if (shift & 4) {
#pragma unroll
        for (int k = 0; k < 5; ++k) w[k] = w[k + 1];
    }
    const u32 bits = (shift & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                      __funnelshift_r(w[3], w[4], bits));
}
#endif

}  // namespace excp
