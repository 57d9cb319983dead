// Norms of rows and their gradients.
//
//   mean and rstd = 1 / sqrt(mean (x - mean)^2 + eps); the RMS form has mean 0          xh = (x - mean) rstd
//   y = xh weight + bias
//   g = dy weight, dx = rstd (g - mean g - xh mean(g xh)) + add  (RMS: without mean g)
//   dweight = sum over rows of dy xh, dbias = sum over rows of dy
//
// A row is held in registers by a group of 32 .. 512 threads, eight columns to a thread and piece: the squares are summed after
// the mean is known, which costs no second read.  Rows past 16384 columns are read again instead.  Sums are fp32.
//
// The gradients of weight and bias are summed in the registers of blocks that walk over the rows; the groups of a block and the
// blocks of a cluster join through (distributed) shared memory in a fixed order, the clusters through a second launch.
// Bound: the bytes.
#include <cooperative_groups.h>

#include "layers.cuh"

namespace cg = cooperative_groups;

namespace excp {
namespace {

constexpr u32 GROUP_MAX = 512;                     // threads of a row at most
constexpr u32 PIECE = 8;                           // columns of a thread at a time

// Sums of two values over a group of `size` threads (a power of two, whole warps), the same in all of them.  `sums`: room of the
// group, two turns of it.
struct GroupSums {
    float2* room;                                  // [2][warps]
    u32 warps, warp, barrier, size, turn = 0;
    __device__ __forceinline__ void operator()(float& a, float& b) {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (warps == 1) return;
        float2* at = room + turn * warps;
        turn ^= 1;                                 // a turn's room is written again only behind the next turn's barrier
        if ((threadIdx.x & 31) == 0) at[warp] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(size) : "memory");
        a = b = 0.f;
        for (u32 w = 0; w < warps; ++w) { const float2 v = at[w]; a += v.x; b += v.y; }
    }
};
__device__ __forceinline__ GroupSums group_sums(float2* room, u32 threads) {
    GroupSums s;
    const u32 group = threadIdx.x / threads;
    s.warps = threads / 32;
    s.room = room + group * 2 * s.warps;
    s.warp = (threadIdx.x - group * threads) / 32;
    s.barrier = 1 + group;
    s.size = threads;
    return s;
}

template <typename T> struct NormArgs {
    const T* x;
    u64 stride, rows;
    u32 cols, threads;                             // threads of a row
    ColumnVector weight, bias;
    float eps;
    u32 rms;
    T* y;
    u64 y_stride;
    float2* stats;                                 // mean, rstd
    Kept kept;                                     // x in 8 bits; codes null: not wanted
};

// PIECES of eight columns to a thread, or 0: the row is read again for each of the three passes.
template <typename T, bool VEC, int PIECES>
__global__ void __launch_bounds__(GROUP_MAX) norm_kernel(const __grid_constant__ NormArgs<T> g) {
    __shared__ float2 room[2 * GROUP_MAX / 32];
    wait_for_previous();
    let_next_start();
    const u32 group = threadIdx.x / g.threads, t = threadIdx.x - group * g.threads, lane = t & 31;
    const u64 row = (u64)blockIdx.x * (blockDim.x / g.threads) + group;
    if (row >= g.rows) return;                     // a whole group
    GroupSums sums = group_sums(room, g.threads);
    const T* x = g.x + row * g.stride;
    const u32 first = t / 32 * 256, step = g.threads * PIECE;
    const float n = (float)g.cols;
    constexpr int HELD = PIECES ? PIECES : 1;
    float v[HELD][8];
    auto each = [&](auto&& f) {                    // f(values, first column of the warp's piece)
        if constexpr (PIECES) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) f(v[p], first + p * step);
        } else {
            for (u32 p0 = 0; p0 < g.cols; p0 += step) {
                load_cols<T, VEC>(x, first + p0, lane, g.cols, v[0]);
                f(v[0], first + p0);
            }
        }
    };
    if constexpr (PIECES) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) load_cols<T, VEC>(x, first + p * step, lane, g.cols, v[p]);
    }
    float mean = 0.f, none = 0.f;
    if (!g.rms) {
        each([&](const float (&a)[8], u32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) mean += a[e];
        });
        sums(mean, none);
        mean /= n;
    }
    float square = 0.f;
    each([&](const float (&a)[8], u32 base) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = a[e] - mean;
            if (lane_col<VEC>(base, lane, e) < g.cols) square = fmaf(d, d, square);
        }
    });
    sums(square, none);
    const float rstd = 1.f / sqrtf(square / n + g.eps);
    if (t == 0 && g.stats) g.stats[row] = make_float2(mean, rstd);
    T* y = g.y + row * g.y_stride;
    each([&](const float (&a)[8], u32 base) {
        if (base >= g.cols) return;                // a whole warp
        float w[8], b[8], r[8];
        load_vector<T, VEC>(g.weight, base, lane, g.cols, 1.f, w);
        load_vector<T, VEC>(g.bias, base, lane, g.cols, 0.f, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = fmaf((a[e] - mean) * rstd, w[e], b[e]);
        if (g.kept.codes) store_kept<VEC>(g.kept, row, base, lane, g.cols, a);
        store_cols<T, VEC>(y, base, lane, g.cols, r);
    });
}

template <typename T> struct GradArgs {
    const T* dy;
    u64 dy_stride;
    const T* x;                                    // or kept
    u64 x_stride;
    Kept kept;
    u64 rows;
    u32 cols, threads;
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
    float2* row_sums;                              // rows that are not held: what the first pass found
};

template <typename T, bool KEPT, bool VEC>
struct RawX {
    Raw<T, VEC> x;
    __device__ __forceinline__ void load(const GradArgs<T>& g, u64 row, u32 base, u32 lane) { x.load(g.x + row * g.x_stride, base, lane, g.cols); }
    __device__ __forceinline__ void values(float (&v)[8]) const { x.values(v); }
};
template <typename T, bool VEC>
struct RawX<T, true, VEC> {
    RawKept<VEC> x;
    __device__ __forceinline__ void load(const GradArgs<T>& g, u64 row, u32 base, u32 lane) { x.load(g.kept, row, base, lane, g.cols); }
    __device__ __forceinline__ void values(float (&v)[8]) const { x.values(v); }
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

template <typename T, bool KEPT, bool VEC, int PIECES>
__global__ void __launch_bounds__(GROUP_MAX, PIECES == 1 ? 2 : 1) norm_grad_kernel(const __grid_constant__ GradArgs<T> g) {
    extern __shared__ float own[];                 // dweight, dbias: the block's
    __shared__ float2 room[2 * GROUP_MAX / 32];
    wait_for_previous();
    let_next_start();
    const u32 groups = blockDim.x / g.threads, group = threadIdx.x / g.threads, t = threadIdx.x - group * g.threads, lane = t & 31;
    GroupSums sums = group_sums(room, g.threads);
    const u32 first = t / 32 * 256, step = g.threads * PIECE;
    const float inv_n = 1.f / (float)g.cols;
    constexpr bool HOLD = PIECES == 1;             // the weight, too
    float w[HOLD ? 1 : 1][8];
    if (HOLD) load_vector<T, VEC>(g.weight, first, lane, g.cols, 1.f, w[0]);
    float dw[PIECES][8] = {}, db[PIECES][8] = {};
    Raw<T, VEC> dy[PIECES];
    RawX<T, KEPT, VEC> x[PIECES];
    float2 st = make_float2(0.f, 0.f);
    const u64 stride = (u64)gridDim.x * groups;
    auto fetch = [&](u64 row) {
        if (row >= g.rows) return;
        st = __ldg(g.stats + row);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            dy[p].load(g.dy + row * g.dy_stride, first + p * step, lane, g.cols);
            x[p].load(g, row, first + p * step, lane);
        }
    };
    u64 row = (u64)blockIdx.x * groups + group;
    fetch(row);
    for (; row < g.rows; row += stride) {
        float d[PIECES][8], xh[PIECES][8], s1 = 0.f, s2 = 0.f;
        const float mean = st.x, rstd = st.y;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            dy[p].values(d[p]);
            x[p].values(xh[p]);
            if (!HOLD) load_vector<T, VEC>(g.weight, first + p * step, lane, g.cols, 1.f, w[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[p][e] = (xh[p][e] - mean) * rstd;
                db[p][e] += d[p][e];               // 0 past the last column
                const float dxh = d[p][e] * xh[p][e];
                dw[p][e] += dxh;
                d[p][e] *= w[0][e];
                s1 += d[p][e];
                s2 = fmaf(dxh, w[0][e], s2);
            }
        }
        fetch(row + stride);                       // on its way while the sums are found
        sums(s1, s2);
        s1 = g.rms ? 0.f : s1 * inv_n;
        s2 *= inv_n;
        if (g.dx) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const u32 base = first + p * step;
                if (base >= g.cols) continue;      // a whole warp
                float r[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] = rstd * (d[p][e] - fmaf(xh[p][e], s2, s1));
                if (g.add) {
                    float a[8];
                    load_cols<T, VEC>(g.add + row * g.add_stride, base, lane, g.cols, a);
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[e] += a[e];
                }
                store_cols<T, VEC>(g.dx + row * g.dx_stride, base, lane, g.cols, r);
            }
        }
    }
    if (!g.dweight && !g.dbias) return;
    // the groups of the block, one after the other
    for (u32 i = 0; i < groups; ++i) {
        __syncthreads();
        if (i != group) continue;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) {
                const u32 c = lane_col<VEC>(first + p * step, lane, e);
                if (c >= g.cols) continue;
                own[c] = i ? own[c] + dw[p][e] : dw[p][e];
                own[g.cols + c] = i ? own[g.cols + c] + db[p][e] : db[p][e];
            }
        }
    }
    const u32 cluster = blockIdx.x / cg::this_cluster().num_blocks();
    if (g.sums) join_cluster(own, 2 * g.cols, 2 * g.cols, g.sums + (u64)cluster * 2 * g.cols, nullptr);
    else join_cluster(own, 2 * g.cols, g.cols, g.dweight, g.dbias);
}

// ---- rows that are not held ---------------------------------------------------------------------------------------------------
// First pass: mean g and mean g xh of every row; a block of GROUP_MAX threads to a row.
template <typename T, bool KEPT, bool VEC>
__global__ void __launch_bounds__(GROUP_MAX) long_sums_kernel(const __grid_constant__ GradArgs<T> g) {
    __shared__ float2 room[2 * GROUP_MAX / 32];
    wait_for_previous();
    let_next_start();
    const u32 lane = threadIdx.x & 31, first = threadIdx.x / 32 * 256, step = GROUP_MAX * PIECE;
    const u64 row = blockIdx.x;
    GroupSums sums = group_sums(room, GROUP_MAX);
    const float2 st = __ldg(g.stats + row);
    float s1 = 0.f, s2 = 0.f;
    for (u32 base = first; base < g.cols; base += step) {
        float d[8], w[8], v[8];
        RawX<T, KEPT, VEC> x;
        x.load(g, row, base, lane);
        load_cols<T, VEC>(g.dy + row * g.dy_stride, base, lane, g.cols, d);
        load_vector<T, VEC>(g.weight, base, lane, g.cols, 1.f, w);
        x.values(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = d[e] * w[e];
            s1 += a;
            s2 = fmaf(a, (v[e] - st.x) * st.y, s2);
        }
    }
    sums(s1, s2);
    if (threadIdx.x == 0) g.row_sums[row] = make_float2(g.rms ? 0.f : s1 / (float)g.cols, s2 / (float)g.cols);
}

// Second pass: strips of 256 columns, a warp to a row.
constexpr u32 LONG_WARPS = 8;
template <typename T, bool KEPT, bool VEC>
__global__ void __launch_bounds__(LONG_WARPS * 32) long_grad_kernel(const __grid_constant__ GradArgs<T> g, u32 row_groups) {
    __shared__ float part[2][LONG_WARPS][256];
    wait_for_previous();
    let_next_start();
    const u32 warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const u32 strip = blockIdx.x / row_groups, rg = blockIdx.x - strip * row_groups, base = strip * 256;
    float dw[8] = {}, db[8] = {}, w[8];
    load_vector<T, VEC>(g.weight, base, lane, g.cols, 1.f, w);
    for (u64 row = (u64)rg * LONG_WARPS + warp; row < g.rows; row += (u64)row_groups * LONG_WARPS) {
        float d[8], v[8], r[8];
        RawX<T, KEPT, VEC> x;
        x.load(g, row, base, lane);
        load_cols<T, VEC>(g.dy + row * g.dy_stride, base, lane, g.cols, d);
        x.values(v);
        const float2 st = __ldg(g.stats + row), sm = g.row_sums[row];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float xh = (v[e] - st.x) * st.y;
            dw[e] = fmaf(d[e], xh, dw[e]);
            db[e] += d[e];
            r[e] = st.y * (d[e] * w[e] - fmaf(xh, sm.y, sm.x));
        }
        if (!g.dx) continue;
        if (g.add) {
            float a[8];
            load_cols<T, VEC>(g.add + row * g.add_stride, base, lane, g.cols, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] += a[e];
        }
        store_cols<T, VEC>(g.dx + row * g.dx_stride, base, lane, g.cols, r);
    }
    if (!g.sums) return;
#pragma unroll
    for (u32 e = 0; e < 8; ++e) {
        part[0][warp][lane_col<VEC>(0, lane, e)] = dw[e];
        part[1][warp][lane_col<VEC>(0, lane, e)] = db[e];
    }
    __syncthreads();
    if (base + threadIdx.x >= g.cols) return;
#pragma unroll
    for (u32 k = 0; k < 2; ++k) {
        float s = 0.f;
#pragma unroll
        for (u32 i = 0; i < LONG_WARPS; ++i) s += part[k][i][threadIdx.x];
        g.sums[((u64)rg * 2 + k) * g.cols + base + threadIdx.x] = s;
    }
}

// ---- how rows are dealt ---------------------------------------------------------------------------------------------------------
bool on16(const void* p, u64 stride_bytes, u64 rows) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows == 1 || (stride_bytes & 15) == 0); }
bool vec(const Matrix& m) { return !m.p || m.dtype == DT_ACT8 || on16(m.p, m.stride * (m.dtype == DT_F32 ? 4 : 2), m.rows); }
bool vec(const ColumnVector& v) { return on16(v.p, 0, 1); }

constexpr u64 HELD_COLS = GROUP_MAX * PIECE * 4;   // longest row that registers hold
u32 threads_of(u64 cols, u32 pieces) {
    u32 t = 32;
    while (t < GROUP_MAX && (u64)t * PIECE * pieces < cols) t *= 2;
    return t;
}

template <typename T, bool VEC, int PIECES>
void norm_launch(cudaStream_t s, NormArgs<T> g) {
    g.threads = PIECES ? threads_of(g.cols, PIECES) : GROUP_MAX;
    // four warps to a block, or one row's
    const u32 block = g.threads > 128 ? g.threads : 128;
    const u64 per = block / g.threads;
    launch_chained(norm_kernel<T, VEC, PIECES>, (u32)((g.rows + per - 1) / per), block, 0, 0, s, g);
}
template <typename T>
void norm_as(cudaStream_t s, const Matrix& x, const ColumnVector& weight, const ColumnVector& bias, float eps, bool rms, const Matrix& y, float* row_stats,
             unsigned char* kept) {
    const NormArgs<T> g{static_cast<const T*>(x.p), x.stride, x.rows, (u32)x.cols, 0, weight, bias, eps, rms, static_cast<T*>(y.p), y.stride,
                        reinterpret_cast<float2*>(row_stats), Kept(kept, x.rows, x.cols)};
    const bool v = vec(x) && vec(y) && vec(weight) && vec(bias);
#define EXCP_N(P) (v ? norm_launch<T, true, P>(s, g) : norm_launch<T, false, P>(s, g))
    if (x.cols <= GROUP_MAX * PIECE) EXCP_N(1);
    else if (x.cols <= GROUP_MAX * PIECE * 2) EXCP_N(2);
    else if (x.cols <= HELD_COLS) EXCP_N(4);
    else EXCP_N(0);
#undef EXCP_N
}

// Blocks of the gradient's kernel, and of a cluster.
struct Deal {
    u32 threads, block, blocks, cluster, sums;     // sums: rows of partial sums; 1: none, written at once
};
Deal deal(int sms, u64 rows, u64 cols) {
    Deal d{};
    const u32 pieces = cols <= GROUP_MAX * PIECE ? 1 : cols <= GROUP_MAX * PIECE * 2 ? 2 : 4;
    d.threads = threads_of(cols, pieces);
    d.block = GROUP_MAX;
    const u64 per = d.block / d.threads, most = (rows + per - 1) / per, full = (u64)sms * (pieces == 1 ? 2 : 1);
    d.blocks = (u32)(most < full ? most : full);
    d.cluster = 1;
    while (d.cluster < 4 && d.cluster < d.blocks) d.cluster *= 2;
    d.blocks = (d.blocks + d.cluster - 1) / d.cluster * d.cluster;
    d.sums = d.blocks / d.cluster;
    return d;
}
u32 long_row_groups(int sms, u64 rows, u64 cols) {
    const u64 strips = (cols + 255) / 256;
    u64 n = ((u64)sms * 4 + strips - 1) / strips;
    const u64 most = (rows + LONG_WARPS - 1) / LONG_WARPS;
    return (u32)(n < most ? n : most);
}

template <typename T, bool KEPT, bool VEC, int PIECES>
void grad_launch(cudaStream_t s, const GradArgs<T>& g, const Deal& d) {
    const u32 smem = (u32)(2 * g.cols * sizeof(float));
    static std::atomic<u64> allowed{0};
    if (smem > 32 * 1024 && !allow_smem(norm_grad_kernel<T, KEPT, VEC, PIECES>, allowed, (u32)(2 * HELD_COLS * sizeof(float)))) return;
    launch_chained(norm_grad_kernel<T, KEPT, VEC, PIECES>, d.blocks, d.block, smem, d.cluster, s, g);
}

template <typename T, bool KEPT, bool VEC>
void grad_as(int sms, cudaStream_t s, GradArgs<T> g, float* scratch) {
    const bool wanted = g.dweight || g.dbias;
    float* const dweight = g.dweight;
    float* const dbias = g.dbias;
    if (g.cols > HELD_COLS) {
        const u32 rg = long_row_groups(sms, g.rows, g.cols);
        g.row_sums = reinterpret_cast<float2*>(scratch);
        g.sums = wanted ? scratch + 2 * g.rows : nullptr;
        launch_chained(long_sums_kernel<T, KEPT, VEC>, (u32)g.rows, GROUP_MAX, 0, 0, s, g);
        launch_chained(long_grad_kernel<T, KEPT, VEC>, (g.cols + 255) / 256 * rg, LONG_WARPS * 32, 0, 0, s, g, rg);
        if (wanted) launch_column_sums(s, g.sums, rg, 2 * (u64)g.cols, g.cols, dweight, dbias);
        return;
    }
    const Deal d = deal(sms, g.rows, g.cols);
    g.threads = d.threads;
    g.sums = wanted && d.sums > 1 ? scratch : nullptr;
    if (g.cols <= GROUP_MAX * PIECE) grad_launch<T, KEPT, VEC, 1>(s, g, d);
    else if (g.cols <= GROUP_MAX * PIECE * 2) grad_launch<T, KEPT, VEC, 2>(s, g, d);
    else grad_launch<T, KEPT, VEC, 4>(s, g, d);
    if (g.sums) launch_column_sums(s, g.sums, d.sums, 2 * (u64)g.cols, g.cols, dweight, dbias);
}

}  // namespace

void launch_layer_norm(int, cudaStream_t s, const Matrix& x, const ColumnVector& weight, const ColumnVector& bias, float eps, bool rms, const Matrix& y,
                       float* row_stats, unsigned char* kept) {
    if (x.dtype == DT_F32) norm_as<float>(s, x, weight, bias, eps, rms, y, row_stats, kept);
    else if (x.dtype == DT_F16) norm_as<__half>(s, x, weight, bias, eps, rms, y, row_stats, kept);
    else norm_as<__nv_bfloat16>(s, x, weight, bias, eps, rms, y, row_stats, kept);
}

u64 layer_norm_grad_scratch(int sms, u64 rows, u64 cols) {
    if (!rows || !cols) return 0;
    if (cols > HELD_COLS) return (2 * rows + (u64)long_row_groups(sms, rows, cols) * 2 * cols) * sizeof(float);
    const Deal d = deal(sms, rows, cols);
    return d.sums > 1 ? d.sums * 2 * cols * sizeof(float) : 0;
}

void launch_layer_norm_grad(int sms, cudaStream_t s, const Matrix& dy, const Matrix& x, const ColumnVector& weight, bool rms, const float* row_stats,
                            const Matrix& add, const Matrix& dx, float* dweight, float* dbias, float* scratch) {
    const bool v = vec(dy) && vec(x) && vec(weight) && vec(add) && vec(dx);
    auto with = [&](auto type) {
        typedef decltype(type) T;
        const GradArgs<T> g{static_cast<const T*>(dy.p), dy.stride, static_cast<const T*>(x.p), x.stride, Kept(x.p, dy.rows, dy.cols), dy.rows, (u32)dy.cols, 0,
                            weight, rms, reinterpret_cast<const float2*>(row_stats), static_cast<const T*>(add.p), add.stride, static_cast<T*>(dx.p),
                            dx.stride, nullptr, dweight, dbias, nullptr};
        if (x.dtype == DT_ACT8) v ? grad_as<T, true, true>(sms, s, g, scratch) : grad_as<T, true, false>(sms, s, g, scratch);
        else v ? grad_as<T, false, true>(sms, s, g, scratch) : grad_as<T, false, false>(sms, s, g, scratch);
    };
    if (dy.dtype == DT_F32) with(float());
    else if (dy.dtype == DT_F16) with(__half());
    else with(__nv_bfloat16());
}

}  // namespace excp
