// Matrices in 8 bits (activations kept for the backward pass), and the gradient through an activation from what was kept.
//
//   blocks of 32 columns: A = max |x|, s = A / 127 rounded up to 8 significant bits, code = nearest whole number of x (1 / s)
//   dpre = dy act'(pre), again = act(pre), dbias = sum over rows of dpre
//
// A warp takes 256 columns of a row, eight to a lane: a block is four lanes' (two shuffles find A).
// Bound: of values in 8 bits and back the bytes (4096 x 11008 bf16 28 us, 5.0 TB/s; back 30 us, 4.6 TB/s).  Of the gradient latency: a value takes 28
// instructions, 13 of them a gelu and its slope, which fill 57 % of the issue slots with 28 % of the warps that an SM could hold; and the blocks of a strip are a
// multiple of its cluster, so that some SMs get three where others get two (4096 x 11008 bf16 from 8 bits, value again: 75 us, 4.2 TB/s; silu 63).
#include <cooperative_groups.h>

#include "layers.cuh"

namespace cg = cooperative_groups;

namespace excp {
namespace {

constexpr u32 SPAN = 256;                          // columns of a warp
constexpr u32 WARPS = 8, THREADS = WARPS * 32;
constexpr u32 ACT_BLOCKS = 3;                      // of the gradient that an SM holds

// A warp takes U pieces of 256 columns, one after the other in the matrix, all fetched before the first is worked on.
template <int U, typename F>
__device__ __forceinline__ void for_pieces(u64 rows, u32 cols, F&& f) {
    const u32 per_row = (cols + SPAN - 1) / SPAN;
    const u64 first = ((u64)blockIdx.x * WARPS + threadIdx.x / 32) * U;
    u64 row;
    u32 piece;
    if ((first >> 32) == 0) {                      // 32 bits: a division of 64 costs as much as eight values
        row = (u32)first / per_row;
        piece = (u32)first - (u32)row * per_row;
    } else {
        row = first / per_row;
        piece = (u32)(first - row * per_row);
    }
    u64 at[U];
    u32 base[U];
    u32 n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = row;
        base[u] = piece * SPAN;
        n += row < rows;
        if (++piece == per_row) { piece = 0; ++row; }
    }
    if (n) f(at, base, n);
}

template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(THREADS) quantize_kernel(const T* __restrict__ x, u64 rows, u32 cols, u64 stride, Kept k) {
    wait_for_previous();
    let_next_start();
    const u32 lane = threadIdx.x & 31;
    for_pieces<U>(rows, cols, [&](const u64 (&row)[U], const u32 (&base)[U], u32 n) {
        Raw<T, VEC> raw[U];
#pragma unroll
        for (u32 u = 0; u < U; ++u) if (u < n) raw[u].load(x + row[u] * stride, base[u], lane, cols);
#pragma unroll
        for (u32 u = 0; u < U; ++u) {
            if (u >= n) break;
            Eight v;
            raw[u].values(v);
            store_kept<VEC>(k, row[u], base[u], lane, v);
        }
    });
}

template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(THREADS) restore_kernel(Kept k, T* out, u64 rows, u32 cols, u64 stride) {
    wait_for_previous();
    let_next_start();
    const u32 lane = threadIdx.x & 31;
    for_pieces<U>(rows, cols, [&](const u64 (&row)[U], const u32 (&base)[U], u32 n) {
        RawKept<VEC> raw[U];
#pragma unroll
        for (u32 u = 0; u < U; ++u) if (u < n) raw[u].load(k, row[u], base[u], lane);
#pragma unroll
        for (u32 u = 0; u < U; ++u) {
            if (u >= n) break;
            Eight v;
            raw[u].values(v);
            store_cols<T, VEC>(out + row[u] * stride, base[u], lane, cols, v);
        }
    });
}

template <typename T> struct Args {
    const T* dy;
    u64 dy_stride;
    const T* pre;                                  // or kept
    u64 pre_stride;
    Kept kept;
    u64 rows;
    u32 cols;
    T* dpre;                                       // null: not wanted
    u64 dpre_stride;
    T* again;                                      // null: not wanted
    u64 again_stride;
    float* sums;                                   // one row of sums per cluster, or dbias itself; null: not wanted
    u32 groups;                                    // blocks that share a strip of columns
};

// A block takes 256 columns and every groups-th set of 8 rows; the column sums of the blocks of a cluster, which share a strip,
// are added through distributed shared memory in the order of the blocks.
template <typename T, bool KEPT, bool VEC, int ACT, int U>
__global__ void __launch_bounds__(THREADS, ACT_BLOCKS) act_grad_kernel(const __grid_constant__ Args<T> g) {
    __shared__ float part[WARPS][SPAN];
    __shared__ float sum[SPAN];
    wait_for_previous();
    let_next_start();
    const u32 warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const u32 strip = blockIdx.x / g.groups, group = blockIdx.x - strip * g.groups, base = strip * SPAN;
    Eight total = {};
    const u64 step = (u64)g.groups * WARPS;
    const u64 row = (u64)group * WARPS + warp;
    const u32 mine = row < g.rows ? (u32)((g.rows - row + step - 1) / step) : 0;       // rows of the warp
    // pointers to the warp's rows, moved by whole steps: products of 64 bits for each would cost as much as the values
    const T* dy_row = g.dy + row * g.dy_stride;
    const T* pre_row = KEPT || ACT == ACT_NONE ? nullptr : g.pre + row * g.pre_stride;
    const u32 per_row = g.kept.blocks;             // blocks of 32 columns
    const unsigned char* code_row = KEPT ? g.kept.codes + row * per_row * A8_BLOCK : nullptr;
    const unsigned short* scale_row = KEPT ? g.kept.scales + row * per_row : nullptr;
    T* dpre_row = g.dpre + row * g.dpre_stride;
    T* again_row = g.again + row * g.again_stride;
    Raw<T, VEC> dy[U], pre[KEPT || ACT == ACT_NONE ? 1 : U];
    RawKept<VEC> kept[KEPT ? U : 1];
    auto fetch = [&](int u) {                      // the next row of the warp
        dy[u].load(dy_row, base, lane, g.cols);
        dy_row += step * g.dy_stride;
        if constexpr (ACT != ACT_NONE) {
            if constexpr (KEPT) {
                kept[u].load(code_row, scale_row, per_row, base, lane);
                code_row += step * per_row * A8_BLOCK;
                scale_row += step * per_row;
            } else {
                pre[u].load(pre_row, base, lane, g.cols);
                pre_row += step * g.pre_stride;
            }
        }
    };
#pragma unroll
    for (u32 u = 0; u < U; ++u) if (u < mine) fetch(u);
    for (u32 at = 0; at < mine; at += U) {
#pragma unroll
        for (u32 u = 0; u < U; ++u) {
            if (at + u >= mine) break;
            Eight d, a, p;
            dy[u].values(d);
            if constexpr (ACT != ACT_NONE) {
                if constexpr (KEPT) kept[u].values(p);
                else pre[u].values(p);
            }
            if (at + u + U < mine) fetch(u);       // on its way while this row is worked on
            if constexpr (ACT != ACT_NONE) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x2 slope;
                    a[i] = act_of<ACT, true>(p[i], slope);
                    d[i] = mul_2(d[i], slope);
                }
                if (g.again) store_cols<T, VEC>(again_row, base, lane, g.cols, a);
                again_row += step * g.again_stride;
            }
            if (g.dpre) store_cols<T, VEC>(dpre_row, base, lane, g.cols, d);
            dpre_row += step * g.dpre_stride;
#pragma unroll
            for (int i = 0; i < 4; ++i) total[i] = add_2(total[i], d[i]);
        }
    }
    if (!g.sums) return;
#pragma unroll
    for (u32 e = 0; e < 8; ++e) part[warp][lane_col<VEC>(0, lane, e)] = e % 2 ? high_2(total[e / 2]) : low_2(total[e / 2]);
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (u32 w = 0; w < WARPS; ++w) s += part[w][threadIdx.x];
    sum[threadIdx.x] = s;
    cg::cluster_group cluster = cg::this_cluster();
    const u32 blocks = cluster.num_blocks(), rank = cluster.block_rank();
    cluster.sync();
    const u32 own = SPAN / blocks, c = rank * own + threadIdx.x;
    if (threadIdx.x < own && base + c < g.cols) {
        float all = 0.f;
        for (u32 b = 0; b < blocks; ++b) all += *cluster.map_shared_rank(&sum[c], b);
        g.sums[(u64)(group / blocks) * g.cols + base + c] = all;
    }
    cluster.sync();                                // the others have read this block's sums
}

// Rows of partial sums -> their sums: 32 columns to a block, eight threads to a column.
__global__ void __launch_bounds__(THREADS) column_sums_kernel(const float* __restrict__ rows, u32 parts, u64 n, u64 split, float* out0, float* out1) {
    __shared__ float part[WARPS][32];
    wait_for_previous();
    let_next_start();
    const u32 warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const u64 c = (u64)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < n) {
#pragma unroll 8
        for (u32 p = warp; p < parts; p += WARPS) s += rows[p * n + c];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp || c >= n) return;
    s = 0.f;
#pragma unroll
    for (u32 w = 0; w < WARPS; ++w) s += part[w][lane];
    if (c < split) { if (out0) out0[c] = s; }
    else if (out1) out1[c - split] = s;
}


template <typename T, bool VEC>
void quantize_as(cudaStream_t s, const Matrix& x, const Kept& k) {
    constexpr int U = sizeof(T) == 4 ? 2 : 4;
    const u64 pieces = x.rows * ((x.cols + SPAN - 1) / SPAN), blocks = (pieces + WARPS * U - 1) / (WARPS * U);
    launch_chained(quantize_kernel<T, VEC, U>, (u32)blocks, THREADS, 0, 0, s, static_cast<const T*>(x.p), x.rows, (u32)x.cols, x.stride, k);
}
template <typename T, bool VEC>
void restore_as(cudaStream_t s, const Kept& k, const Matrix& y) {
    constexpr int U = 4;
    const u64 pieces = y.rows * ((y.cols + SPAN - 1) / SPAN), blocks = (pieces + WARPS * U - 1) / (WARPS * U);
    launch_chained(restore_kernel<T, VEC, U>, (u32)blocks, THREADS, 0, 0, s, k, static_cast<T*>(y.p), y.rows, (u32)y.cols, y.stride);
}

// How the rows of a strip of columns are split: blocks in all, and blocks of a cluster.  Three blocks to an SM where there are
// rows enough (two to a warp); up to eight blocks join within one cluster, so that a second launch is not needed.
struct Split {
    u32 groups, cluster;
};
Split act_split(int sms, u64 rows, u64 cols) {
    const u64 strips = (cols + SPAN - 1) / SPAN, most = (rows + 2 * WARPS - 1) / (2 * WARPS);
    u64 groups = (u64)sms * ACT_BLOCKS / strips;            // no more than find room at once
    if (groups > most) groups = most;
    if (groups > 8 && rows <= 8 * 6 * WARPS) groups = 8;         // six rows to a warp cost less than the second launch
    if (groups < 1) groups = 1;
    Split r{1, 1};
    while (r.cluster * 2 <= groups && r.cluster < (groups <= 8 ? 8u : 4u)) r.cluster *= 2;
    r.groups = (u32)(groups / r.cluster * r.cluster);
    return r;
}

template <typename T, bool KEPT, bool VEC, int ACT>
void act_grad_launch(cudaStream_t s, const Args<T>& g, const Split& p) {
    const u32 strips = (g.cols + SPAN - 1) / SPAN;
    launch_chained(act_grad_kernel<T, KEPT, VEC, ACT, ACT == ACT_NONE ? 6 : 2>, strips * p.groups, THREADS, 0, g.sums ? p.cluster : 0, s, g);
}

template <typename T>
void act_grad_as(int sms, cudaStream_t s, int act, const Matrix& dy, const Matrix& pre, const Matrix& dpre, const Matrix& again, float* dbias, float* scratch) {
    const Split p = act_split(sms, dy.rows, dy.cols);
    const u32 rows_of_sums = p.groups / p.cluster;
    const bool kept = pre.dtype == DT_ACT8;
    const Args<T> g{static_cast<const T*>(dy.p), dy.stride, static_cast<const T*>(pre.p), pre.stride, Kept(pre.p, dy.rows, dy.cols), dy.rows, (u32)dy.cols,
                    static_cast<T*>(dpre.p), dpre.stride, static_cast<T*>(again.p), again.stride, dbias ? (rows_of_sums > 1 ? scratch : dbias) : nullptr, p.groups};
    const bool v = in_words(dy) && in_words(pre) && in_words(dpre) && in_words(again);
#define EXCP_AG(ACT) (kept ? (v ? act_grad_launch<T, true, true, ACT>(s, g, p) : act_grad_launch<T, true, false, ACT>(s, g, p)) \
                           : (v ? act_grad_launch<T, false, true, ACT>(s, g, p) : act_grad_launch<T, false, false, ACT>(s, g, p)))
    if (act == ACT_GELU) EXCP_AG(ACT_GELU);
    else if (act == ACT_GELU_TANH) EXCP_AG(ACT_GELU_TANH);
    else if (act == ACT_SILU) EXCP_AG(ACT_SILU);
    else if (v) act_grad_launch<T, false, true, ACT_NONE>(s, g, p);
    else act_grad_launch<T, false, false, ACT_NONE>(s, g, p);
#undef EXCP_AG
    if (dbias && rows_of_sums > 1) launch_column_sums(s, scratch, rows_of_sums, dy.cols, dy.cols, dbias, nullptr);
}

}  // namespace

void launch_column_sums(cudaStream_t s, const float* rows, u32 parts, u64 n, u64 split, float* out0, float* out1) {
    launch_chained(column_sums_kernel, (u32)((n + 31) / 32), THREADS, 0, 0, s, rows, parts, n, split, out0, out1);
}

void launch_act8_quantize(cudaStream_t s, const Matrix& x, unsigned char* packed) {
    const Kept k(packed, x.rows, x.cols);
#define EXCP_Q(T) (in_words(x) ? quantize_as<T, true>(s, x, k) : quantize_as<T, false>(s, x, k))
    if (x.dtype == DT_F32) EXCP_Q(float);
    else if (x.dtype == DT_F16) EXCP_Q(__half);
    else EXCP_Q(__nv_bfloat16);
#undef EXCP_Q
}

void launch_act8_restore(cudaStream_t s, const unsigned char* packed, const Matrix& y) {
    const Kept k(const_cast<unsigned char*>(packed), y.rows, y.cols);
#define EXCP_R(T) (in_words(y) ? restore_as<T, true>(s, k, y) : restore_as<T, false>(s, k, y))
    if (y.dtype == DT_F32) EXCP_R(float);
    else if (y.dtype == DT_F16) EXCP_R(__half);
    else EXCP_R(__nv_bfloat16);
#undef EXCP_R
}

u64 act_grad_scratch(int sms, u64 rows, u64 cols) {
    if (!rows || !cols) return 0;
    const Split p = act_split(sms, rows, cols);
    return p.groups == p.cluster ? 0 : p.groups / p.cluster * cols * sizeof(float);
}

void launch_act_grad(int sms, cudaStream_t s, int act, const Matrix& dy, const Matrix& pre, const Matrix& dpre, const Matrix& again, float* dbias, float* scratch) {
#define EXCP_A(T) act_grad_as<T>(sms, s, act, dy, pre, dpre, again, dbias, scratch)
    if (dy.dtype == DT_F32) EXCP_A(float);
    else if (dy.dtype == DT_F16) EXCP_A(__half);
    else EXCP_A(__nv_bfloat16);
#undef EXCP_A
}

}  // namespace excp
