// Product of two microscaled 4-bit matrices: y[a row, b row] = scales * sum over columns (+ bias), fp32 sums.
//
// Tensor cores: tcgen05.mma on packed 4-bit floats with their block scales (64 columns per instruction), fp32
// accumulators in tensor memory.  The packed layout is the one the tensor core reads, tile by tile: a stage of
// the pipeline is a handful of contiguous bulk copies (codes of the M rows, codes of the N rows, scales of
// both), no address pattern, no tensor map.
//
// Roles: warps 0..3 write the result, warp 4 fetches, warp 5 issues the matrix instructions.
// Every wait is bounded; where one runs out the block raises the handle's flag, lets its copies land and leaves.
#include "score.cuh"
#include "tcgen05.cuh"

namespace excp {
namespace {

constexpr int THREADS = 192;
constexpr int STAGES = 4;
constexpr u32 A_CODES = MX4_ROWS * 128;
constexpr u64 DRAIN_NS = 100000000ull;             // a copy in flight lands within microseconds

struct MatmulArgs {
    Mx4Operand m, n;             // the operands on the M side (128 rows per tile) and on the N side
    u32 col_tiles;
    u32 nt;                      // rows of n per block: a multiple of 8, at most 256
    void* y;
    u64 sm, sn;                  // strides of y along the rows of m and of n
    const float* bias;
    u32 bias_on_m;
    u32 stage_bytes, tmem_cols;
    u64 wait_ns;
    u32* flag;
};

struct Shared {
    unsigned long long full[STAGES], empty[STAGES], done;
    u32 tmem;
    volatile u32 abort;
};

// One thread waits for phase `parity` of `bar`; false when the limit has passed or another role gave up.
__device__ __forceinline__ bool wait_one(Shared* sh, unsigned long long* bar, u32 parity, u64 limit_ns, u32* flag) {
    if (limit_ns) {
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        const u64 t0 = global_ns();
        while (!sh->abort) {
            if (mbar_try_wait(bar, parity)) return true;
            if (global_ns() - t0 > limit_ns) break;
        }
    }
    if (!sh->abort) {
        sh->abort = 1;
        *reinterpret_cast<volatile u32*>(flag) = 1;
        __threadfence_system();
    }
    return false;
}
// The same without raising anything: for letting one's own work land before leaving.
__device__ __forceinline__ void drain_one(unsigned long long* bar, u32 parity) {
    const u64 t0 = global_ns();
    while (!mbar_try_wait(bar, parity) && global_ns() - t0 < DRAIN_NS) {}
}

template <int DT>
__device__ __forceinline__ void put(void* y, u64 at, float v) {
    wput(static_cast<typename ElemOf<DT>::type*>(y), at, v);
}

template <int FMT, int DT>
__global__ void __launch_bounds__(THREADS, 1) matmul_kernel(const __grid_constant__ MatmulArgs g) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared sh;
    // the swizzle goes by address: stages start on 1024 bytes
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    constexpr u32 PIECES = mx4_pieces(FMT), SB = mx4_scale_bytes(FMT);
    const u32 warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const u32 n_tiles = (u32)((g.n.rows + g.nt - 1) / g.nt);
    const u32 mt = blockIdx.x / n_tiles, n0 = (blockIdx.x - mt * n_tiles) * g.nt;
    // the N side spans one or two row tiles of its matrix
    const u32 nt0 = n0 / MX4_ROWS;
    const u32 parts = g.nt > MX4_ROWS && (u64)(nt0 + 1) * MX4_ROWS < g.n.rows ? 2 : 1;

    const u32 base = smem_u32(smem);
    const u32 b_codes = A_CODES, scales = A_CODES + g.nt * 128;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        mbar_init(&sh.done, 1);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == 5) tm_alloc(&sh.tmem, g.tmem_cols);
    tm_fence_before();
    __syncthreads();
    tm_fence_after();
    const u32 tmem = sh.tmem;

    if (warp == 4 && lane == 0) {
        const u32 hm = mx4_tile_height(g.m.rows, mt);
        const u32 h0 = mx4_tile_height(g.n.rows, nt0), h1 = parts == 2 ? mx4_tile_height(g.n.rows, nt0 + 1) : 0;
        const u32 bytes = (hm + h0 + h1) * 128 + (1 + parts) * SB;
        const unsigned char* pm = g.m.p + mx4_tile_offset(g.m.rows, g.col_tiles, FMT, mt, 0);
        const unsigned char* p0 = g.n.p + mx4_tile_offset(g.n.rows, g.col_tiles, FMT, nt0, 0);
        const unsigned char* p1 = parts == 2 ? g.n.p + mx4_tile_offset(g.n.rows, g.col_tiles, FMT, nt0 + 1, 0) : nullptr;
        u32 issued = 0;
        for (u32 k = 0; k < g.col_tiles; ++k) {
            const u32 s = k % STAGES, turn = k / STAGES;
            if (turn && !wait_one(&sh, &sh.empty[s], (turn - 1) & 1, g.wait_ns, g.flag)) break;
            unsigned char* st = smem + s * g.stage_bytes;
            mbar_arrive_expect_tx(&sh.full[s], bytes);
            bulk_g2s(st, pm, hm * 128, &sh.full[s]);
            bulk_g2s(st + scales, pm + hm * 128, SB, &sh.full[s]);
            bulk_g2s(st + b_codes, p0, h0 * 128, &sh.full[s]);
            bulk_g2s(st + scales + SB, p0 + h0 * 128, SB, &sh.full[s]);
            pm += hm * 128 + SB;
            p0 += h0 * 128 + SB;
            if (parts == 2) {
                bulk_g2s(st + b_codes + A_CODES, p1, h1 * 128, &sh.full[s]);
                bulk_g2s(st + scales + 2 * SB, p1 + h1 * 128, SB, &sh.full[s]);
                p1 += h1 * 128 + SB;
            }
            ++issued;
        }
        // no copy may be in flight when the block leaves (a matrix instruction need not have waited for it)
        for (u32 k = issued > STAGES ? issued - STAGES : 0; k < issued; ++k) drain_one(&sh.full[k % STAGES], (k / STAGES) & 1);
    } else if (warp == 5 && lane == 0) {
        const u32 idesc0 = (1u << 7) | (1u << 10) | ((g.nt >> 3) << 17) | (FMT == MX4_E8M0_32 ? 1u << 23 : 0u) | (8u << 24);
        const u32 b_groups = (g.nt + MX4_ROWS - 1) / MX4_ROWS;
        const u32 sf_cols = PIECES * 4 * (1 + b_groups);
        bool ok = true;
        for (u32 k = 0; k < g.col_tiles; ++k) {
            const u32 s = k % STAGES;
            if (!wait_one(&sh, &sh.full[s], (k / STAGES) & 1, g.wait_ns, g.flag)) { ok = false; break; }
            tm_fence_after();
            const u32 st = base + s * g.stage_bytes;
            // each stage has scale columns of its own, free again when the stage is
            const u32 sa = tmem + g.nt + s * sf_cols, sb = sa + PIECES * 4;
            for (u32 j = 0; j < PIECES; ++j) {
                tm_copy_scales(sa + j * 4, desc_scales(st + scales + j * MX4_PIECE));
                for (u32 q = 0; q < parts; ++q)
                    tm_copy_scales(sb + j * 4 * b_groups + q * 4, desc_scales(st + scales + (1 + q) * SB + j * MX4_PIECE));
            }
            const u64 da = desc_swizzled(st), db = desc_swizzled(st + b_codes);
#pragma unroll
            for (u32 i = 0; i < 4; ++i) {             // 64 columns = 32 bytes of codes each
                if (FMT == MX4_E4M3_16) {
                    tm_mma_block16(tmem, da + 2 * i, db + 2 * i, idesc0, sa + i * 4, sb + i * 4 * b_groups, k || i);
                } else {
                    const u32 half = (i & 1) * 2;     // a piece serves two instructions: its bytes 0, 1, then 2, 3
                    const u32 j = i >> 1;
                    tm_mma_block32(tmem, da + 2 * i, db + 2 * i, idesc0 | (half << 4) | (half << 29), sa + j * 4, sb + j * 4 * b_groups, k || i);
                }
            }
            tm_commit(&sh.empty[s]);
        }
        tm_commit(&sh.done);
        if (!ok) drain_one(&sh.done, 0);
    } else if (warp < 4) {
        const bool ok = g.col_tiles == 0 || __all_sync(0xffffffffu, wait_one(&sh, &sh.done, 0, g.wait_ns, g.flag));
        tm_fence_after();
        if (ok) {
            const float alpha = (g.m.scale ? __ldg(g.m.scale) : 1.f) * (g.n.scale ? __ldg(g.n.scale) : 1.f);
            const u64 m = (u64)mt * MX4_ROWS + warp * 32 + lane;
            const float bias_m = g.bias && g.bias_on_m && m < g.m.rows ? __ldg(g.bias + m) : 0.f;
            for (u32 c = 0; c < g.nt; c += 8) {
                u32 v[8];
                tm_load8(tmem + ((warp * 32) << 16) + c, v);
                tm_wait_load();
#pragma unroll
                for (u32 i = 0; i < 8; ++i) {
                    const u64 n = (u64)n0 + c + i;
                    if (n >= g.n.rows || m >= g.m.rows) continue;
                    float f = g.col_tiles ? __uint_as_float(v[i]) * alpha : 0.f;
                    if (g.bias) f += g.bias_on_m ? bias_m : __ldg(g.bias + n);
                    put<DT>(g.y, m * g.sm + n * g.sn, f);
                }
            }
        }
        tm_fence_before();
    }
    __syncwarp();
    __syncthreads();
    if (warp == 5) tm_dealloc(tmem, g.tmem_cols);
}

template <int FMT, int DT>
bool launch_as(cudaStream_t s, const MatmulArgs& g) {
    const u32 smem = g.stage_bytes * STAGES + 1024;
    if (cudaFuncSetAttribute(matmul_kernel<FMT, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
    const u32 grid = (u32)((g.n.rows + g.nt - 1) / g.nt) * mx4_row_tiles(g.m.rows);
    matmul_kernel<FMT, DT><<<grid, THREADS, smem, s>>>(g);
    return true;
}

}  // namespace

bool launch_mx4_matmul(int sms, cudaStream_t s, const Mx4Operand& a, const Mx4Operand& b, u64 cols, int fmt,
                       const Mx4Result& r, u64 wait_ns, u32* flag) {
    if (cols && a.rows > MX4_ROWS && b.rows > MX4_ROWS) return launch_mx4_matmul_wide(sms, s, a, b, cols, fmt, r, wait_ns, flag);
    MatmulArgs g{};
    // few rows of a: they go to the N side, whose width the tensor core takes in steps of 8
    const bool swap = a.rows <= MX4_ROWS;
    g.m = swap ? b : a;
    g.n = swap ? a : b;
    g.col_tiles = mx4_col_tiles(cols);
    g.nt = g.n.rows > 2 * MX4_ROWS ? 2 * MX4_ROWS : (u32)((g.n.rows + 7) & ~7ull);
    g.y = r.y;
    g.sm = swap ? 1 : r.stride;
    g.sn = swap ? r.stride : 1;
    g.bias = r.bias;
    g.bias_on_m = swap;
    const u32 groups = (g.nt + MX4_ROWS - 1) / MX4_ROWS;
    g.stage_bytes = A_CODES + g.nt * 128 + (1 + groups) * (u32)mx4_scale_bytes(fmt);
    const u32 need = g.nt + STAGES * (u32)mx4_pieces(fmt) * 4 * (1 + groups);
    g.tmem_cols = 32;
    while (g.tmem_cols < need) g.tmem_cols *= 2;
    g.wait_ns = wait_ns;
    g.flag = flag;
#define EXCP_MM(DT) (fmt == MX4_E4M3_16 ? launch_as<MX4_E4M3_16, DT>(s, g) : launch_as<MX4_E8M0_32, DT>(s, g))
    return r.dtype == DT_F32 ? EXCP_MM(DT_F32) : r.dtype == DT_F16 ? EXCP_MM(DT_F16) : EXCP_MM(DT_BF16);
#undef EXCP_MM
}

}  // namespace excp
