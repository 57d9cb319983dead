// Norms of rows and their gradients.
//
//   mean and rstd = 1 / sqrt(mean (x - mean)^2 + eps); the RMS form has mean 0          xh = (x - mean) rstd
//   y = xh weight + bias
//   g = dy weight, dx = rstd (g - mean g - xh mean(g xh)) + add  (RMS: without mean g)
//   dweight = sum over rows of dy xh, dbias = sum over rows of dy
// Lanes past the last column have xh 0: (0 - mean) rstd can be infinite, and would spoil the sum of g xh although g is 0 there.
//
// A row is held in registers, as it lies in memory, by a group of 32 .. 512 threads, eight columns to a thread and piece: the squares are
// summed after the mean is known, which costs no second read.  With few rows a thread has one piece; where there are rows enough, as few threads as hold a
// row in four: a warp up to 1024 columns (no barrier), 128 threads at 4096.  A warp has 256 columns of one row at a time, so of rows shorter than that
// some of its lanes have none.  (8192 x 4096 bf16: 512 threads to a row 85 us, 256 threads with the rows in a ring in shared memory 45, 128 threads
// 36.)  Rows past what registers hold are read again.  Sums are fp32.
//
// The gradient of few rows is one kernel: blocks walk over the rows and sum the gradients of weight and bias in registers.  With
// many rows that costs two barriers a row and half the registers (8192 x 4096 bf16 from 8 bits 103 us); there, dx is one kernel as above,
// and the sums are another, which reads dy and x again: strips of 256 columns, a warp to a row (59 us together).  Either way the sums of
// a cluster's blocks join through distributed shared memory in a fixed order, the clusters' through a further launch.
// Bound: the bytes; of the forward pass the latency of a row's two sums, behind which nothing of the next row is on its way (issue slots 46 % busy).
#include <cooperative_groups.h>

#include "layers.cuh"

namespace cg = cooperative_groups;

namespace excp {
namespace {

constexpr u32 GROUP_MAX = 512;                     // threads of a row at most
constexpr u32 PIECE = 8;                           // columns of a thread at a time

// Sums of one or two values over a group of `size` threads (a power of two, whole warps), the same in all of them.  `room`: of the
// group, two turns of it.
struct GroupSums {
    float2* room;                                  // [2][warps]
    u32 warps, warp, barrier, size, turn = 0;
    __device__ __forceinline__ float2* meet(float a, float b) {            // behind the barrier: the warps' sums
        float2* at = room + turn;
        turn ^= warps;                             // a turn's room is written again only behind the next turn's barrier
        if ((threadIdx.x & 31) == 0) at[warp] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(size) : "memory");
        return at + (threadIdx.x & (warps - 1));
    }
    __device__ __forceinline__ void operator()(float& a, float& b) {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (warps == 1) return;
        const float2 v = *meet(a, b);
        a = v.x;
        b = v.y;
#pragma unroll
        for (u32 o = 1; o < GROUP_MAX / 32; o *= 2) {
            if (o >= warps) break;
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
    }
    __device__ __forceinline__ float operator()(float a) {
#pragma unroll
        for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if (warps == 1) return a;
        a = meet(a, 0.f)->x;
#pragma unroll
        for (u32 o = 1; o < GROUP_MAX / 32; o *= 2) {
            if (o >= warps) break;
            a += __shfl_xor_sync(0xffffffffu, a, o);
        }
        return a;
    }
};
__device__ __forceinline__ GroupSums group_sums(float2* room, u32 threads, u32 threads_log) {
    GroupSums s;
    const u32 group = threadIdx.x >> threads_log;
    s.warps = threads / 32;
    s.room = room + group * 2 * s.warps;
    s.warp = (threadIdx.x & (threads - 1)) / 32;
    s.barrier = 1 + group;
    s.size = threads;
    return s;
}

// 1 / sqrt(squares / n + eps).  It moves a whole row alike, so of 32-bit rows each step is rounded to the nearest.  What is rounded to 16 bits
// afterwards takes a product with 1 / n and the approximate root (1.4 * 2^-24 off instead of 1.0; the exact ones: 8192 x 4096 bf16 35.7 -> 36.8 us).
template <typename T>
__device__ __forceinline__ float reciprocal_root(float squares, float n, float eps) {
    if constexpr (sizeof(T) == 4) return __frsqrt_rn(squares / n + eps);
    else return rsqrtf(fmaf(squares, 1.f / n, eps));
}

template <typename T> struct NormArgs {
    const T* x;
    u64 stride, rows;
    u32 cols, threads, threads_log, rows_log;      // threads of a row; rows of a block
    ColumnVector weight, bias;
    float eps;
    u32 rms;
    T* y;
    u64 y_stride;
    float2* stats;                                 // mean, rstd
    Kept kept;                                     // x in 8 bits; codes null: not wanted
};

// PIECES of eight columns to a thread, or 0: the row is read again for each of the three passes.
template <int PIECES> constexpr int block_of() { return PIECES < 2 ? (int)GROUP_MAX : 128; }      // threads of a block at most

template <typename T, bool VEC, int PIECES>
__global__ void __launch_bounds__(block_of<PIECES>(), PIECES < 2 ? 2 : 5) norm_kernel(const __grid_constant__ NormArgs<T> g) {
    __shared__ float2 room[2 * GROUP_MAX / 32];
    wait_for_previous();
    let_next_start();
    const u32 group = threadIdx.x >> g.threads_log, t = threadIdx.x & (g.threads - 1), lane = t & 31;
    const u64 row = ((u64)blockIdx.x << g.rows_log) + group;
    if (row >= g.rows) return;                     // a whole group
    GroupSums sums = group_sums(room, g.threads, g.threads_log);
    const T* x = g.x + row * g.stride;
    const u32 first = t / 32 * 256, step = g.threads * PIECE;
    const float n = (float)g.cols;
    Raw<T, VEC> held[PIECES ? PIECES : 1];
    auto each = [&](auto&& f) {                    // f(values, first column of the warp's piece)
        if constexpr (PIECES) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                if (p && first + p * step >= g.cols) break;      // a whole warp
                Eight v;
                held[p].values(v);
                f(v, first + p * step);
            }
        } else {
            for (u32 base = first; base < g.cols; base += step) {
                Eight v;
                load_cols<T, VEC>(x, base, lane, g.cols, v);
                f(v, base);
            }
        }
    };
    if constexpr (PIECES) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) if (!p || first + p * step < g.cols) held[p].load(x, first + p * step, lane, g.cols);
    }
    float mean = 0.f;
    if (!g.rms) {
        f32x2 sum = 0;
        each([&](const Eight& a, u32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = add_2(sum, a[i]);
        });
        mean = sums(low_2(sum) + high_2(sum)) / n;      // divided: the mean of equal values is that value
    }
    const f32x2 minus_mean = both_2(-mean);
    f32x2 squares = 0;
    each([&](const Eight& a, u32 base) {
        f32x2 piece = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x2 d = add_2(a[i], minus_mean);
            if (!VEC) {
                if (lane_col<VEC>(base, lane, 2 * i) >= g.cols) d &= ~0xffffffffull;
                if (lane_col<VEC>(base, lane, 2 * i + 1) >= g.cols) d &= 0xffffffffull;
            }
            piece = fma_2(d, d, piece);
        }
        if (!VEC || base + lane * 8 < g.cols) squares = add_2(squares, piece);         // VEC: a lane's eight are in or out
    });
    const float rstd = reciprocal_root<T>(sums(low_2(squares) + high_2(squares)), n, g.eps);
    if (t == 0 && g.stats) g.stats[row] = make_float2(mean, rstd);
    T* y = g.y + row * g.y_stride;
    const f32x2 both_rstd = both_2(rstd);
    each([&](const Eight& a, u32 base) {
        if (base >= g.cols) return;                // a whole warp
        Eight w, b, r;
        load_vector<T, VEC>(g.weight, base, lane, g.cols, 1.f, w);
        load_vector<T, VEC>(g.bias, base, lane, g.cols, 0.f, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = fma_2(mul_2(add_2(a[i], minus_mean), both_rstd), w[i], b[i]);
        if (g.kept.codes) store_kept<VEC>(g.kept, row, base, lane, a);
        store_cols<T, VEC>(y, base, lane, g.cols, r);
    });
}

// The same for many rows in 16-byte words, with all that can be known when it is compiled: THREADS of a row (so that a piece's place
// is a constant), and what vectors there are (VECTORS: 1 the weight, 2 the bias too, both of T).  Half the instructions of the kernel above
// (8192 x 4096 bf16: 43 us there, 36 here, 46 with x in 8 bits; 16384 x 1024 25 and 16).
__host__ __device__ constexpr int rows_block(int threads) { return threads > 128 ? threads : 128; }
__host__ __device__ constexpr u32 const_log(u32 v) { return v <= 1 ? 0 : 1 + const_log(v / 2); }
template <typename T, int PIECES, int THREADS, int VECTORS>
__global__ void __launch_bounds__(rows_block(THREADS), 512 / rows_block(THREADS)) norm_rows_kernel(const __grid_constant__ NormArgs<T> g) {
    constexpr u32 BLOCK = rows_block(THREADS), STEP = THREADS * PIECE, LOG = const_log(THREADS);
    __shared__ float2 room[2 * BLOCK / 32];
    wait_for_previous();
    let_next_start();
    const u32 t = threadIdx.x % THREADS, lane = t & 31, at = t * PIECE;
    const u64 row = (u64)blockIdx.x * (BLOCK / THREADS) + threadIdx.x / THREADS;
    if (row >= g.rows) return;                     // a whole group
    GroupSums sums = group_sums(room, THREADS, LOG);
    const T* x = g.x + row * g.stride + at;
    const float n = (float)g.cols;
    Raw<T, true> raw[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) raw[p].load_at(x + p * STEP, at + p * STEP < g.cols);
    Eight v[PIECES];
    f32x2 sum = 0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        raw[p].values(v[p]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = add_2(sum, v[p][i]);
    }
    float mean = 0.f;
    if (!g.rms) mean = sums(low_2(sum) + high_2(sum)) / n;       // divided: the mean of equal values is that value
    const f32x2 minus_mean = both_2(-mean);
    f32x2 squares = 0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        f32x2 piece = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 d = add_2(v[p][i], minus_mean);
            piece = fma_2(d, d, piece);
        }
        if (at + p * STEP < g.cols) squares = add_2(squares, piece);
    }
    const float rstd = reciprocal_root<T>(sums(low_2(squares) + high_2(squares)), n, g.eps);
    if (t == 0 && g.stats) g.stats[row] = make_float2(mean, rstd);
    const f32x2 both_rstd = both_2(rstd);
    T* y = g.y + row * g.y_stride + at;
    const T* weight = static_cast<const T*>(g.weight.p) + at;
    const T* bias = static_cast<const T*>(g.bias.p) + at;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const bool there = at + p * STEP < g.cols;
        if (g.kept.codes && p * STEP + at - lane * PIECE < g.cols) store_kept<true>(g.kept, row, p * STEP + at - lane * PIECE, lane, v[p]);
        if (!there) continue;
        Raw<T, true> w, b;
        Eight we, be;
        w.template load_at<false>(weight + p * STEP, true);
        w.values(we);
        if (VECTORS == 2) {
            b.template load_at<false>(bias + p * STEP, true);
            b.values(be);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 xh = mul_2(add_2(v[p][i], minus_mean), both_rstd);
            v[p][i] = VECTORS == 2 ? fma_2(xh, we[i], be[i]) : mul_2(xh, we[i]);
        }
        store_eight(y + p * STEP, v[p]);
    }
}

template <typename T> struct GradArgs {
    const T* dy;
    u64 dy_stride;
    const T* x;                                    // or kept
    u64 x_stride;
    Kept kept;
    u64 rows;
    u32 cols, threads, threads_log, rows_log;
    ColumnVector weight;
    u32 rms;
    const float2* stats;
    const T* add;                                  // null: none
    u64 add_stride;
    T* dx;
    u64 dx_stride;
    float* sums;                                   // per cluster dweight, then dbias, or null
    float* dweight;                                // where there is one cluster alone
    float* dbias;
    u32 groups;                                    // of the sums alone: blocks that share a strip of columns
};

template <typename T, bool KEPT, bool VEC>
struct RawX {
    Raw<T, VEC> x;
    __device__ __forceinline__ void load(const GradArgs<T>& g, u64 row, u32 base, u32 lane) { x.load(g.x + row * g.x_stride, base, lane, g.cols); }
    __device__ __forceinline__ void values(Eight& v) const { x.values(v); }
};
template <typename T, bool VEC>
struct RawX<T, true, VEC> {
    RawKept<VEC> x;
    __device__ __forceinline__ void load(const GradArgs<T>& g, u64 row, u32 base, u32 lane) { x.load(g.kept, row, base, lane); }
    __device__ __forceinline__ void values(Eight& v) const { x.values(v); }
};

// Adds what the blocks of a cluster have in own[0..n) and writes it: column c < split to out0[c], the others to out1.
__device__ __forceinline__ void join_cluster(float* own, u32 n, u32 split, float* out0, float* out1) {
    cg::cluster_group cluster = cg::this_cluster();
    const u32 blocks = cluster.num_blocks(), rank = cluster.block_rank();
    cluster.sync();
    for (u32 c = rank * blockDim.x + threadIdx.x; c < n; c += blocks * blockDim.x) {
        float all = 0.f;
        for (u32 b = 0; b < blocks; ++b) all += *cluster.map_shared_rank(own + c, b);
        if (c < split) { if (out0) out0[c] = all; }
        else if (out1) out1[c - split] = all;
    }
    cluster.sync();                                // the others have read this block's
}

template <typename T, bool KEPT, bool VEC>
__global__ void __launch_bounds__(GROUP_MAX, 1) norm_grad_kernel(const __grid_constant__ GradArgs<T> g) {
    extern __shared__ float own[];                 // dweight, dbias: the block's
    __shared__ float2 room[2 * GROUP_MAX / 32];
    wait_for_previous();
    let_next_start();
    const u32 groups = 1u << g.rows_log, group = threadIdx.x >> g.threads_log, t = threadIdx.x & (g.threads - 1), lane = t & 31;
    GroupSums sums = group_sums(room, g.threads, g.threads_log);
    const u32 base = t / 32 * 256;                 // a thread has one piece
    const float inv_n = 1.f / (float)g.cols;
    Eight dw = {}, db = {};
    Raw<T, VEC> dy;
    RawX<T, KEPT, VEC> x;
    float2 st = make_float2(0.f, 0.f);
    const u64 stride = (u64)gridDim.x * groups;
    auto fetch = [&](u64 row) {
        if (row >= g.rows) return;
        st = __ldg(g.stats + row);
        dy.load(g.dy + row * g.dy_stride, base, lane, g.cols);
        x.load(g, row, base, lane);
    };
    u64 row = (u64)blockIdx.x * groups + group;
    fetch(row);
    for (; row < g.rows; row += stride) {
        Eight d, xh, w;
        f32x2 s1 = 0, s2 = 0;
        const f32x2 minus_mean = both_2(-st.x), rstd = both_2(st.y);
        dy.values(d);
        x.values(xh);
        load_vector<T, VEC>(g.weight, base, lane, g.cols, 1.f, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xh[i] = mul_2(add_2(xh[i], minus_mean), where_column<VEC>(base, lane, g.cols, i, st.y));
            db[i] = add_2(db[i], d[i]);            // 0 past the last column
            dw[i] = fma_2(d[i], xh[i], dw[i]);
            d[i] = mul_2(d[i], w[i]);
            s1 = add_2(s1, d[i]);
            s2 = fma_2(d[i], xh[i], s2);
        }
        fetch(row + stride);                       // on its way while the sums are found
        float m1 = low_2(s1) + high_2(s1), m2 = low_2(s2) + high_2(s2);
        sums(m1, m2);
        if (base < g.cols) {                       // a whole warp
            const f32x2 minus_m1 = both_2(g.rms ? 0.f : -m1 * inv_n), minus_m2 = both_2(-m2 * inv_n);
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = mul_2(rstd, add_2(d[i], fma_2(xh[i], minus_m2, minus_m1)));
            if (g.add) {
                Eight a;
                load_cols<T, VEC>(g.add + row * g.add_stride, base, lane, g.cols, a);
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = add_2(d[i], a[i]);
            }
            store_cols<T, VEC>(g.dx + row * g.dx_stride, base, lane, g.cols, d);
        }
    }
    // the groups of the block, one after the other
    for (u32 i = 0; i < groups; ++i) {
        __syncthreads();
        if (i != group) continue;
#pragma unroll
        for (u32 e = 0; e < 8; ++e) {
            const u32 c = lane_col<VEC>(base, lane, e);
            if (c >= g.cols) continue;
            const float a = e % 2 ? high_2(dw[e / 2]) : low_2(dw[e / 2]), b = e % 2 ? high_2(db[e / 2]) : low_2(db[e / 2]);
            own[c] = i ? own[c] + a : a;
            own[g.cols + c] = i ? own[g.cols + c] + b : b;
        }
    }
    const u32 cluster = blockIdx.x / cg::this_cluster().num_blocks();
    if (g.sums) join_cluster(own, 2 * g.cols, 2 * g.cols, g.sums + (u64)cluster * 2 * g.cols, nullptr);
    else join_cluster(own, 2 * g.cols, g.cols, g.dweight, g.dbias);
}

// ---- many rows ------------------------------------------------------------------------------------------------------------------
// dx alone.  PIECES as above.
template <typename T, bool KEPT, bool VEC, int PIECES>
__global__ void __launch_bounds__(PIECES == 2 ? 128 : GROUP_MAX, PIECES == 2 ? 6 : PIECES == 1 ? 2 : 1) norm_dx_kernel(const __grid_constant__ GradArgs<T> g) {
    __shared__ float2 room[2 * GROUP_MAX / 32];
    wait_for_previous();
    let_next_start();
    const u32 group = threadIdx.x >> g.threads_log, t = threadIdx.x & (g.threads - 1), lane = t & 31;
    const u64 row = ((u64)blockIdx.x << g.rows_log) + group;
    if (row >= g.rows) return;                     // a whole group
    GroupSums sums = group_sums(room, g.threads, g.threads_log);
    const u32 first = t / 32 * 256, step = g.threads * PIECE;
    const float inv_n = 1.f / (float)g.cols;
    const float2 st = __ldg(g.stats + row);
    const f32x2 minus_mean = both_2(-st.x), rstd = both_2(st.y);
    constexpr int HELD = PIECES ? PIECES : 1;
    Eight held_g[HELD], held_xh[HELD];
    Raw<T, VEC> dy[HELD];
    RawX<T, KEPT, VEC> x[HELD];
    auto load = [&](int p, u32 base) {
        dy[p].load(g.dy + row * g.dy_stride, base, lane, g.cols);
        x[p].load(g, row, base, lane);
    };
    auto take = [&](int p, u32 base) {
        Eight w;
        dy[p].values(held_g[p]);
        x[p].values(held_xh[p]);
        load_vector<T, VEC>(g.weight, base, lane, g.cols, 1.f, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            held_xh[p][i] = mul_2(add_2(held_xh[p][i], minus_mean), where_column<VEC>(base, lane, g.cols, i, st.y));
            held_g[p][i] = mul_2(held_g[p][i], w[i]);            // 0 past the last column
        }
    };
    auto each = [&](auto&& f) {                    // f(g, xh, first column of the warp's piece)
        if constexpr (PIECES) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                if (p && first + p * step >= g.cols) break;      // a whole warp
                f(held_g[p], held_xh[p], first + p * step);
            }
        } else {
            for (u32 base = first; base < g.cols; base += step) {
                load(0, base);
                take(0, base);
                f(held_g[0], held_xh[0], base);
            }
        }
    };
    if constexpr (PIECES) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) if (!p || first + p * step < g.cols) load(p, first + p * step);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) if (!p || first + p * step < g.cols) take(p, first + p * step);
    }
    f32x2 s1 = 0, s2 = 0;
    each([&](const Eight& d, const Eight& xh, u32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s1 = add_2(s1, d[i]);
            s2 = fma_2(d[i], xh[i], s2);
        }
    });
    float m1 = low_2(s1) + high_2(s1), m2 = low_2(s2) + high_2(s2);
    sums(m1, m2);
    const f32x2 minus_m1 = both_2(g.rms ? 0.f : -m1 * inv_n), minus_m2 = both_2(-m2 * inv_n);
    each([&](const Eight& d, const Eight& xh, u32 base) {
        if (base >= g.cols) return;                // a whole warp
        Eight r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = mul_2(rstd, add_2(d[i], fma_2(xh[i], minus_m2, minus_m1)));
        if (g.add) {
            Eight a;
            load_cols<T, VEC>(g.add + row * g.add_stride, base, lane, g.cols, a);
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = add_2(r[i], a[i]);
        }
        store_cols<T, VEC>(g.dx + row * g.dx_stride, base, lane, g.cols, r);
    });
}

// The same as above (norm_rows_kernel), with a weight of T.  8192 x 4096 bf16 35 us (5.7 TB/s), fp32 4096 x 4096 32 us (6.3 TB/s).
template <typename T, bool KEPT, int PIECES, int THREADS>
__global__ void __launch_bounds__(rows_block(THREADS), 512 / rows_block(THREADS)) norm_dx_rows_kernel(const __grid_constant__ GradArgs<T> g) {
    constexpr u32 BLOCK = rows_block(THREADS), STEP = THREADS * PIECE, LOG = const_log(THREADS);
    __shared__ float2 room[2 * BLOCK / 32];
    wait_for_previous();
    let_next_start();
    const u32 t = threadIdx.x % THREADS, at = t * PIECE;
    const u64 row = (u64)blockIdx.x * (BLOCK / THREADS) + threadIdx.x / THREADS;
    if (row >= g.rows) return;                     // a whole group
    GroupSums sums = group_sums(room, THREADS, LOG);
    const T* dy = g.dy + row * g.dy_stride + at;
    const float inv_n = 1.f / (float)g.cols;
    Raw<T, true> raw[PIECES], x[KEPT ? 1 : PIECES];
    uint2 codes[KEPT ? PIECES : 1];
    float scale[KEPT ? PIECES : 1];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) raw[p].load_at(dy + p * STEP, at + p * STEP < g.cols);
    if constexpr (KEPT) {
        const unsigned char* c = g.kept.codes + row * g.kept.blocks * A8_BLOCK + at;
        const unsigned short* s = g.kept.scales + row * g.kept.blocks + at / A8_BLOCK;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const bool there = at + p * STEP < g.cols;
            codes[p] = there ? __ldg(reinterpret_cast<const uint2*>(c + p * STEP)) : make_uint2(0u, 0u);
            scale[p] = there ? __uint_as_float((u32)__ldg(s + p * STEP / A8_BLOCK) << 16) : 0.f;
        }
    } else {
        const T* from = g.x + row * g.x_stride + at;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) x[p].load_at(from + p * STEP, at + p * STEP < g.cols);
    }
    const float2 st = __ldg(g.stats + row);
    const f32x2 minus_mean = both_2(-st.x), rstd = both_2(st.y);
    const T* weight = static_cast<const T*>(g.weight.p) + at;
    Eight d[PIECES], xh[PIECES];
    f32x2 s1 = 0, s2 = 0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        Raw<T, true> w;
        Eight we;
        w.template load_at<false>(weight + p * STEP, at + p * STEP < g.cols);
        const f32x2 here = both_2(at + p * STEP < g.cols ? st.y : 0.f);
        w.values(we);
        raw[p].values(d[p]);
        if constexpr (KEPT) a8_eight(codes[p].x, codes[p].y, scale[p], xh[p]);
        else x[p].values(xh[p]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xh[p][i] = mul_2(add_2(xh[p][i], minus_mean), here);
            d[p][i] = mul_2(d[p][i], we[i]);       // 0 past the last column
            s1 = add_2(s1, d[p][i]);
            s2 = fma_2(d[p][i], xh[p][i], s2);
        }
    }
    float m1 = low_2(s1) + high_2(s1), m2 = low_2(s2) + high_2(s2);
    sums(m1, m2);
    const f32x2 minus_m1 = both_2(g.rms ? 0.f : -m1 * inv_n), minus_m2 = both_2(-m2 * inv_n);
    T* dx = g.dx + row * g.dx_stride + at;
    const T* add = g.add ? g.add + row * g.add_stride + at : nullptr;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        if (at + p * STEP >= g.cols) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) d[p][i] = mul_2(rstd, add_2(d[p][i], fma_2(xh[p][i], minus_m2, minus_m1)));
        if (add) {
            Raw<T, true> r;
            Eight a;
            r.load_at(add + p * STEP, true);
            r.values(a);
#pragma unroll
            for (int i = 0; i < 4; ++i) d[p][i] = add_2(d[p][i], a[i]);
        }
        store_eight(dx + p * STEP, d[p]);
    }
}

// dweight and dbias alone: a block takes 256 columns and every groups-th set of 8 rows, a warp a row, COLUMN_ROWS of them on their way.
// (512 columns to a warp: 8192 x 4096 38 us against 35, 16384 x 1024 37 against 24.)
constexpr int COLUMN_ROWS = 4;                     // (8192 x 4096: two rows 34 us, four 24)
constexpr u32 SUM_WARPS = 8, SUM_BLOCKS = 3;       // blocks that an SM holds
template <typename T, bool KEPT, bool VEC>
__global__ void __launch_bounds__(SUM_WARPS * 32, SUM_BLOCKS) norm_columns_kernel(const __grid_constant__ GradArgs<T> g) {
    constexpr int U = COLUMN_ROWS;
    constexpr u32 SPAN = 256;
    __shared__ float part[SUM_WARPS][256];
    __shared__ float own[2 * SPAN];
    wait_for_previous();
    let_next_start();
    const u32 warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const u32 strip = blockIdx.x / g.groups, group = blockIdx.x - strip * g.groups, base = strip * SPAN;
    const u64 step = (u64)g.groups * SUM_WARPS, row = (u64)group * SUM_WARPS + warp;
    const u32 mine = row < g.rows ? (u32)((g.rows - row + step - 1) / step) : 0;       // rows of the warp
    // pointers to the warp's rows, moved by whole steps: products of 64 bits for each would cost as much as the values
    const T* dy_row = g.dy + row * g.dy_stride;
    const T* x_row = KEPT ? nullptr : g.x + row * g.x_stride;
    const u32 per_row = g.kept.blocks;             // blocks of 32 columns
    const unsigned char* code_row = KEPT ? g.kept.codes + row * per_row * A8_BLOCK : nullptr;
    const unsigned short* scale_row = KEPT ? g.kept.scales + row * per_row : nullptr;
    const float2* stat = g.stats + row;
    const u64 dy_step = step * g.dy_stride, x_step = step * g.x_stride, code_step = step * per_row * A8_BLOCK, scale_step = step * per_row;
    Raw<T, VEC> dy[U];
    RawX<T, KEPT, VEC> x[U];
    float2 st[U];
    auto fetch = [&](int u) {                      // the next row of the warp
        dy[u].load(dy_row, base, lane, g.cols);
        dy_row += dy_step;
        if constexpr (KEPT) {
            x[u].x.load(code_row, scale_row, per_row, base, lane);
            code_row += code_step;
            scale_row += scale_step;
        } else {
            x[u].x.load(x_row, base, lane, g.cols);
            x_row += x_step;
        }
        st[u] = __ldg(stat);
        stat += step;
    };
    Eight dw = {}, db = {};
#pragma unroll
    for (u32 u = 0; u < U; ++u) if (u < mine) fetch(u);
    for (u32 at = 0; at < mine; at += U) {
#pragma unroll
        for (u32 u = 0; u < U; ++u) {
            if (at + u >= mine) break;
            Eight d, xh;
            const f32x2 minus_mean = both_2(-st[u].x), rstd = both_2(st[u].y);
            dy[u].values(d);
            x[u].values(xh);
            if (at + u + U < mine) fetch(u);       // on its way while this row is worked on
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                db[k] = add_2(db[k], d[k]);
                dw[k] = fma_2(d[k], mul_2(add_2(xh[k], minus_mean), rstd), dw[k]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (u32 e = 0; e < 8; ++e) {
            const f32x2 v = k ? db[e / 2] : dw[e / 2];
            part[warp][lane_col<VEC>(0, lane, e)] = e % 2 ? high_2(v) : low_2(v);
        }
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (u32 i = 0; i < SUM_WARPS; ++i) s += part[i][threadIdx.x];
        own[k * 256 + threadIdx.x] = s;
        __syncthreads();
    }
    cg::cluster_group cluster = cg::this_cluster();
    const u32 blocks = cluster.num_blocks(), rank = cluster.block_rank();
    cluster.sync();
    for (u32 c = rank * 256 + threadIdx.x; c < 2 * SPAN; c += blocks * 256) {
        const u32 k = c / SPAN, col = base + c % SPAN;
        float all = 0.f;
        for (u32 b = 0; b < blocks; ++b) all += *cluster.map_shared_rank(own + c, b);
        if (col >= g.cols) continue;
        if (g.sums) g.sums[((u64)(group / blocks) * 2 + k) * g.cols + col] = all;
        else if (k == 0 && g.dweight) g.dweight[col] = all;
        else if (k == 1 && g.dbias) g.dbias[col] = all;
    }
    cluster.sync();                                // the others have read this block's sums
}

// ---- how rows are dealt ---------------------------------------------------------------------------------------------------------

// How a row is dealt: pieces of a thread (0: too long to be held), threads, threads of a block.
struct Rows {
    u32 pieces, threads, block;
};
// Few rows: as many threads to a row as it has words of eight columns.  Many, or long ones: as few as can hold it.
Rows rows_of(int sms, u64 rows, u64 cols, u32 most_pieces, u32 most_threads) {
    if (cols > (u64)most_threads * PIECE * most_pieces) return Rows{0, GROUP_MAX, GROUP_MAX};
    Rows r{1, 32, 128};
    const bool many = rows > (u64)sms * 4 || cols > GROUP_MAX * PIECE;
    while ((u64)r.threads * PIECE * r.pieces < cols) {
        if (many && r.pieces < most_pieces) r.pieces *= 2;
        else r.threads *= 2;
    }
    if (r.threads > r.block) r.block = r.threads;
    return r;
}
u32 log2_of(u32 v) { return v <= 1 ? 0 : 1 + log2_of(v / 2); }
template <typename T, bool VEC, int PIECES>
void norm_launch(cudaStream_t s, NormArgs<T> g, const Rows& r) {
    g.threads = r.threads;
    g.threads_log = log2_of(r.threads);
    g.rows_log = log2_of(r.block / r.threads);
    launch_chained(norm_kernel<T, VEC, PIECES>, (u32)((g.rows + (1u << g.rows_log) - 1) >> g.rows_log), r.block, 0, 0, s, g);
}
// The kernels of many rows: four words to a thread (eight: 8192 x 4096 bf16 47 us against 36), as few threads as hold a row, or two
// words where a warp holds it so.  False where they do not take it.
template <typename T> constexpr int code_of() { return std::is_same<T, float>::value ? DT_F32 : std::is_same<T, __half>::value ? DT_F16 : DT_BF16; }
constexpr u64 ROWS_COLS = 512 * PIECE * 4;
template <typename T, int PIECES, int THREADS>
void norm_rows_launch(cudaStream_t s, const NormArgs<T>& g) {
    constexpr u32 block = rows_block(THREADS), per = block / THREADS;
    const u32 blocks = (u32)((g.rows + per - 1) / per);
    if (g.bias.p) launch_chained(norm_rows_kernel<T, PIECES, THREADS, 2>, blocks, block, 0, 0, s, g);
    else launch_chained(norm_rows_kernel<T, PIECES, THREADS, 1>, blocks, block, 0, 0, s, g);
}
template <typename T>
bool norm_rows(int sms, cudaStream_t s, const NormArgs<T>& g) {
    if (g.rows <= (u64)sms * 4 || g.cols > ROWS_COLS || !g.weight.p || g.weight.dtype != code_of<T>() || (g.bias.p && g.bias.dtype != code_of<T>())) return false;
    if (g.cols <= 32 * PIECE * 2) norm_rows_launch<T, 2, 32>(s, g);
    else if (g.cols <= 32 * PIECE * 4) norm_rows_launch<T, 4, 32>(s, g);
    else if (g.cols <= 64 * PIECE * 4) norm_rows_launch<T, 4, 64>(s, g);
    else if (g.cols <= 128 * PIECE * 4) norm_rows_launch<T, 4, 128>(s, g);
    else if (g.cols <= 256 * PIECE * 4) norm_rows_launch<T, 4, 256>(s, g);
    else norm_rows_launch<T, 4, 512>(s, g);
    return true;
}
template <typename T, bool KEPT, int PIECES, int THREADS>
void dx_rows_launch(cudaStream_t s, const GradArgs<T>& g) {
    constexpr u32 block = rows_block(THREADS), per = block / THREADS;
    launch_chained(norm_dx_rows_kernel<T, KEPT, PIECES, THREADS>, (u32)((g.rows + per - 1) / per), block, 0, 0, s, g);
}
template <typename T, bool KEPT>
bool dx_rows(int sms, cudaStream_t s, const GradArgs<T>& g) {
    if (g.rows <= (u64)sms * 4 || g.cols > ROWS_COLS || !g.weight.p || g.weight.dtype != code_of<T>()) return false;
    if (g.cols <= 32 * PIECE * 2) dx_rows_launch<T, KEPT, 2, 32>(s, g);
    else if (g.cols <= 32 * PIECE * 4) dx_rows_launch<T, KEPT, 4, 32>(s, g);
    else if (g.cols <= 64 * PIECE * 4) dx_rows_launch<T, KEPT, 4, 64>(s, g);
    else if (g.cols <= 128 * PIECE * 4) dx_rows_launch<T, KEPT, 4, 128>(s, g);
    else if (g.cols <= 256 * PIECE * 4) dx_rows_launch<T, KEPT, 4, 256>(s, g);
    else dx_rows_launch<T, KEPT, 4, 512>(s, g);
    return true;
}
template <typename T, bool VEC>
void norm_as(int sms, cudaStream_t s, const NormArgs<T>& g) {
    if constexpr (VEC) if (norm_rows<T>(sms, s, g)) return;
    const Rows r = rows_of(sms, g.rows, g.cols, 8, 128);
    if (r.pieces == 0) norm_launch<T, VEC, 0>(s, g, r);
    else if (r.pieces == 1) norm_launch<T, VEC, 1>(s, g, r);
    else if (r.pieces == 2) norm_launch<T, VEC, 2>(s, g, r);
    else if (r.pieces == 4) norm_launch<T, VEC, 4>(s, g, r);
    else norm_launch<T, VEC, 8>(s, g, r);
}

// The gradient in one kernel: while no group of threads has more than three rows.
constexpr u64 FUSED_COLS = GROUP_MAX * PIECE;
struct Deal {
    Rows rows;
    u32 blocks, cluster;
};
u32 cluster_of(u64 blocks) { return blocks >= 4 ? 4 : blocks >= 2 ? 2 : 1; }
bool deal_fused(int sms, u64 rows, u64 cols, Deal& d) {
    if (cols > FUSED_COLS) return false;
    d.rows = Rows{1, 32, GROUP_MAX};
    while ((u64)d.rows.threads * PIECE < cols) d.rows.threads *= 2;
    const u64 per = GROUP_MAX / d.rows.threads, most = (rows + per - 1) / per;
    if (most > (u64)sms * 3) return false;
    const u64 blocks = most < (u64)sms ? most : (u64)sms;
    d.cluster = cluster_of(blocks);
    d.blocks = (u32)((blocks + d.cluster - 1) / d.cluster * d.cluster);
    return true;
}
// The sums alone: blocks of a strip, and of a cluster.
Deal deal_sums(int sms, u64 rows, u64 cols) {
    Deal d{};
    const u64 strips = (cols + 255) / 256, most = (rows + 2 * SUM_WARPS - 1) / (2 * SUM_WARPS);
    u64 groups = (u64)sms * SUM_BLOCKS / strips;       // no more than find room at once
    if (groups > most) groups = most;
    if (groups < 1) groups = 1;
    d.cluster = cluster_of(groups);
    d.blocks = (u32)(groups / d.cluster * d.cluster);
    return d;
}

template <typename T, bool KEPT, bool VEC, int PIECES>
void dx_launch(cudaStream_t s, GradArgs<T> g, const Rows& r) {
    g.threads = r.threads;
    g.threads_log = log2_of(r.threads);
    g.rows_log = log2_of(r.block / r.threads);
    launch_chained(norm_dx_kernel<T, KEPT, VEC, PIECES>, (u32)((g.rows + (1u << g.rows_log) - 1) >> g.rows_log), r.block, 0, 0, s, g);
}

template <typename T, bool KEPT, bool VEC>
void grad_as(int sms, cudaStream_t s, GradArgs<T> g, float* scratch) {
    float* const dweight = g.dweight;
    float* const dbias = g.dbias;
    const bool wanted = dweight || dbias;
    u32 sums = 1;                                  // rows of partial sums
    Deal d;
    if (wanted && g.dx && deal_fused(sms, g.rows, g.cols, d)) {
        sums = d.blocks / d.cluster;
        g.sums = sums > 1 ? scratch : nullptr;
        g.threads = d.rows.threads;
        g.threads_log = log2_of(g.threads);
        g.rows_log = log2_of(GROUP_MAX / g.threads);
        launch_chained(norm_grad_kernel<T, KEPT, VEC>, d.blocks, GROUP_MAX, (u32)(2 * g.cols * sizeof(float)), d.cluster, s, g);
    } else {
        if (wanted) {                              // first: dx may take dy's place
            d = deal_sums(sms, g.rows, g.cols);
            sums = d.blocks / d.cluster;
            g.sums = sums > 1 ? scratch : nullptr;
            g.groups = d.blocks;
            launch_chained(norm_columns_kernel<T, KEPT, VEC>, (g.cols + 255) / 256 * d.blocks, SUM_WARPS * 32, 0, d.cluster, s, g);
        }
        bool done = !g.dx;
        if constexpr (VEC) done = done || dx_rows<T, KEPT>(sms, s, g);
        if (!done) {
            const Rows r = rows_of(sms, g.rows, g.cols, 4, GROUP_MAX);
            if (r.pieces == 0) dx_launch<T, KEPT, VEC, 0>(s, g, r);
            else if (r.pieces == 1) dx_launch<T, KEPT, VEC, 1>(s, g, r);
            else if (r.pieces == 2) dx_launch<T, KEPT, VEC, 2>(s, g, r);
            else dx_launch<T, KEPT, VEC, 4>(s, g, r);
        }
    }
    if (sums > 1) launch_column_sums(s, scratch, sums, 2 * (u64)g.cols, g.cols, dweight, dbias);
}

}  // namespace

void launch_layer_norm(int sms, cudaStream_t s, const Matrix& x, const ColumnVector& weight, const ColumnVector& bias, float eps, bool rms, const Matrix& y,
                       float* row_stats, unsigned char* kept) {
    const bool v = in_words(x) && in_words(y) && in_words(weight) && in_words(bias);
    auto with = [&](auto type) {
        typedef decltype(type) T;
        const NormArgs<T> g{static_cast<const T*>(x.p), x.stride, x.rows, (u32)x.cols, 0, 0, 0, weight, bias, eps, rms, static_cast<T*>(y.p), y.stride,
                            reinterpret_cast<float2*>(row_stats), Kept(kept, x.rows, x.cols)};
        v ? norm_as<T, true>(sms, s, g) : norm_as<T, false>(sms, s, g);
    };
    if (x.dtype == DT_F32) with(float());
    else if (x.dtype == DT_F16) with(__half());
    else with(__nv_bfloat16());
}

u64 layer_norm_grad_scratch(int sms, u64 rows, u64 cols) {
    if (!rows || !cols) return 0;
    Deal d, fused;
    d = deal_sums(sms, rows, cols);
    u32 sums = d.blocks / d.cluster;
    if (deal_fused(sms, rows, cols, fused) && fused.blocks / fused.cluster > sums) sums = fused.blocks / fused.cluster;
    return sums > 1 ? sums * 2 * cols * sizeof(float) : 0;
}

void launch_layer_norm_grad(int sms, cudaStream_t s, const Matrix& dy, const Matrix& x, const ColumnVector& weight, bool rms, const float* row_stats,
                            const Matrix& add, const Matrix& dx, float* dweight, float* dbias, float* scratch) {
    const bool v = in_words(dy) && in_words(x) && in_words(weight) && in_words(add) && in_words(dx);
    auto with = [&](auto type) {
        typedef decltype(type) T;
        const GradArgs<T> g{static_cast<const T*>(dy.p), dy.stride, static_cast<const T*>(x.p), x.stride, Kept(x.p, dy.rows, dy.cols), dy.rows, (u32)dy.cols, 0, 0, 0,
                            weight, rms, reinterpret_cast<const float2*>(row_stats), static_cast<const T*>(add.p), add.stride, static_cast<T*>(dx.p),
                            dx.stride, nullptr, dweight, dbias, 0};
        if (x.dtype == DT_ACT8) v ? grad_as<T, true, true>(sms, s, g, scratch) : grad_as<T, true, false>(sms, s, g, scratch);
        else v ? grad_as<T, false, true>(sms, s, g, scratch) : grad_as<T, false, false>(sms, s, g, scratch);
    };
    if (dy.dtype == DT_F32) with(float());
    else if (dy.dtype == DT_F16) with(__half());
    else with(__nv_bfloat16());
}

}  // namespace excp
