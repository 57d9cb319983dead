// Product of two microscaled 4-bit matrices, many rows on both sides (see mx4_matmul.cu for few).
//
// Bound: the tensor cores, and close behind them shared memory: 4-bit operands run through the matrix pipe so fast
// (128 x 256 x 64 in 128 cycles) that a CTA alone would write and read 200 bytes of tiles per cycle.  A pair of CTAs
// therefore works on one 256 x 256 tile (tcgen05 cta_group::2): each holds 128 rows of a and half the rows of b,
// which takes a third off the traffic.
//
// Persistent pairs: pair p computes tiles p, p + pairs, ...  Roles in each CTA: warps 0..7 write the result, warp 8
// fetches (contiguous bulk copies, the packed layout is the tensor core's), warp 9 of the even CTA issues the matrix
// instructions, warps 10..13 bring the block scales to tensor memory.  The accumulator (256 columns of tensor memory) is read
// into registers in one go and handed back before it is converted and written, so that the next tile waits for a
// few hundred cycles only.
// Every wait is bounded; where one runs out the CTA raises the handle's flag, lets its copies land and leaves (the
// partner's waits run out in turn).
#include "score.cuh"
#include "tcgen05.cuh"

namespace excp {
namespace {

constexpr int STORE_WARPS = 8;
constexpr int SCALE_WARPS = 4;
constexpr int THREADS = (STORE_WARPS + 2 + SCALE_WARPS) * 32;
constexpr u32 CODES = MX4_ROWS * 128;              // codes of one operand tile
constexpr u32 SPAN = 2 * MX4_ROWS;                 // rows of a and of b per pair
constexpr u32 GROUP = 8;                           // tiles of a that are visited before the next tile of b
constexpr u64 DRAIN_NS = 100000000ull;

template <int FMT> __host__ __device__ constexpr int stages() { return FMT == MX4_E4M3_16 ? 5 : 6; }
template <int FMT> __host__ __device__ constexpr u32 stage_bytes() { return 2 * CODES + 3 * mx4_scale_bytes(FMT); }

struct WideArgs {
    Mx4Operand m, n;                               // on the M side (TMEM lanes) and the N side (columns)
    u32 col_tiles, m_tiles, n_tiles;
    void* y;
    u64 stride;
    const float* bias;                             // per row of b (the operand on the contiguous side of y)
    u32 wide_store;                                // rows of y start on 32 bytes
    u64 wait_ns;
    u32* flag;
};

template <int FMT>
struct Shared {
    unsigned long long full[stages<FMT>()];        // own copies have landed
    unsigned long long ready[stages<FMT>()];       // even CTA: both CTAs' have, and the scales are in tensor memory
    unsigned long long empty[stages<FMT>()];       // the stage has been multiplied
    unsigned long long acc_full, acc_empty;
    u32 tmem;
    volatile u32 abort;
};

template <typename S>
__device__ __forceinline__ bool wait_one(S* sh, unsigned long long* bar, u32 parity, const WideArgs& g) {
    if (g.wait_ns) {
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        const u64 t0 = global_ns();
        while (!sh->abort) {
            if (mbar_try_wait(bar, parity)) return true;
            if (global_ns() - t0 > g.wait_ns) break;
        }
    }
    if (!sh->abort) {
        sh->abort = 1;
        *reinterpret_cast<volatile u32*>(g.flag) = 1;
        __threadfence_system();
    }
    return false;
}
__device__ __forceinline__ void drain_one(unsigned long long* bar, u32 parity) {
    const u64 t0 = global_ns();
    while (!mbar_try_wait(bar, parity) && global_ns() - t0 < DRAIN_NS) {}
}

// Tile `t` of the pairs' common order: GROUP tiles of m for one tile of n, then the next tile of n.
__device__ __forceinline__ void place(const WideArgs& g, u32 t, u32& mt, u32& nt) {
    const u32 per_group = GROUP * g.n_tiles;
    const u32 group = t / per_group, inside = t - group * per_group;
    const u32 rows = min(GROUP, g.m_tiles - group * GROUP);
    nt = inside / rows;
    mt = group * GROUP + inside - nt * rows;
}

template <int DT> __device__ __forceinline__ u32 two(float a, float b) {
    if (DT == DT_F16) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const u32*>(&h); }
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const u32*>(&h);
}
__device__ __forceinline__ void store32(void* p, const u32 v[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// The first `cols` of a row's results, packed in WORDS words.
template <typename T, u32 WORDS>
__device__ __forceinline__ void put_row(T* y, const u32 (&w)[WORDS], u32 cols, u32 wide_store) {
    constexpr u32 PER = 4 / sizeof(T);
#pragma unroll
    for (u32 i = 0; i < WORDS; i += 8) {
        if (wide_store && (i + 8) * PER <= cols) {
            const u32 v[8] = {w[i], w[i + 1], w[i + 2], w[i + 3], w[i + 4], w[i + 5], w[i + 6], w[i + 7]};
            store32(y + i * PER, v);
        } else {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) {
                if constexpr (PER == 2) {
                    unsigned short* h = reinterpret_cast<unsigned short*>(y) + (i + e) * 2;
                    if ((i + e) * 2 < cols) h[0] = (unsigned short)(w[i + e] & 0xffffu);
                    if ((i + e) * 2 + 1 < cols) h[1] = (unsigned short)(w[i + e] >> 16);
                } else {
                    if (i + e < cols) reinterpret_cast<u32*>(y)[i + e] = w[i + e];
                }
            }
        }
    }
}

template <int FMT, int DT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) wide_kernel(const __grid_constant__ WideArgs g) {
    typedef typename ElemOf<DT>::type T;
    constexpr int STAGES = stages<FMT>();
    constexpr u32 PIECES = mx4_pieces(FMT), SB = mx4_scale_bytes(FMT), STAGE = stage_bytes<FMT>();
    constexpr u32 SF_COLS = PIECES * 12;           // scales of a stage in tensor memory: 128 rows of m, 256 of n
    constexpr u32 TMEM_COLS = 512;
    static_assert(SPAN + STAGES * SF_COLS <= TMEM_COLS, "tensor memory");
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared<FMT> sh;
    // the swizzle goes by address: stages start on 1024 bytes (the same offset in both CTAs)
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const u32 base = smem_u32(smem);
    const u32 warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const u32 rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const u32 tiles = g.m_tiles * g.n_tiles;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.ready[s], 2 * SCALE_WARPS); mbar_init(&sh.empty[s], 1); }
        mbar_init(&sh.acc_full, 1);
        mbar_init(&sh.acc_empty, 2 * STORE_WARPS);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == STORE_WARPS + 1) tm2_alloc(&sh.tmem, TMEM_COLS);
    tm_fence_before();
    __syncthreads();
    cluster_barrier();                             // the partner's barriers are ready
    tm_fence_after();
    const u32 tmem = sh.tmem;

    if (warp == STORE_WARPS && lane == 0) {
        u32 step = 0;                              // stages filled so far
        bool ok = true;
        for (u32 t = pair; ok && t < tiles; t += pairs) {
            u32 mt, nt;
            place(g, t, mt, nt);
            const u32 rm = 2 * mt + rank, rn = 2 * nt;
            // row tiles past the end are not fetched: their rows' results are not written
            const bool has_m = (u64)rm * MX4_ROWS < g.m.rows, has_n1 = (u64)(rn + 1) * MX4_ROWS < g.n.rows, has_own = rank == 0 || has_n1;
            const u32 hm = has_m ? mx4_tile_height(g.m.rows, rm) : 0;
            const u32 h0 = mx4_tile_height(g.n.rows, rn), h1 = has_n1 ? mx4_tile_height(g.n.rows, rn + 1) : 0;
            const u32 own = rank == 0 ? h0 : h1;
            const unsigned char* pm = has_m ? g.m.p + mx4_tile_offset(g.m.rows, g.col_tiles, FMT, rm, 0) : nullptr;
            const unsigned char* p0 = g.n.p + mx4_tile_offset(g.n.rows, g.col_tiles, FMT, rn, 0);
            const unsigned char* p1 = has_n1 ? g.n.p + mx4_tile_offset(g.n.rows, g.col_tiles, FMT, rn + 1, 0) : nullptr;
            const u32 bytes = hm * 128 + (has_m ? SB : 0) + own * 128 + SB + (has_n1 ? SB : 0);
            for (u32 k = 0; k < g.col_tiles; ++k, ++step) {
                const u32 s = step % STAGES, turn = step / STAGES;
                if (turn && !wait_one(&sh, &sh.empty[s], (turn - 1) & 1, g)) { ok = false; break; }
                unsigned char* st = smem + s * STAGE;
                unsigned long long* bar = &sh.full[s];
                mbar_arrive_expect_tx(bar, bytes);
                if (has_m) {
                    bulk_g2s(st, pm, hm * 128, bar);
                    bulk_g2s(st + 2 * CODES, pm + hm * 128, SB, bar);
                    pm += hm * 128 + SB;
                }
                if (has_own) bulk_g2s(st + CODES, rank == 0 ? p0 : p1, own * 128, bar);
                bulk_g2s(st + 2 * CODES + SB, p0 + h0 * 128, SB, bar);      // the scales of all of n's rows go to both CTAs
                p0 += h0 * 128 + SB;
                if (has_n1) {
                    bulk_g2s(st + 2 * CODES + 2 * SB, p1 + h1 * 128, SB, bar);
                    p1 += h1 * 128 + SB;
                }
            }
        }
        // no copy may be in flight when the CTA leaves
        for (u32 k = step > STAGES ? step - STAGES : 0; k < step; ++k) drain_one(&sh.full[k % STAGES], (k / STAGES) & 1);
    } else if (warp == STORE_WARPS + 1 && lane == 0) {
        u32 step = 0, turn_acc = 0;
        bool ok = true;
        if (rank == 0) {
            constexpr u32 IDESC = (1u << 7) | (1u << 10) | ((SPAN >> 3) << 17) | (FMT == MX4_E8M0_32 ? 1u << 23 : 0u) | ((SPAN >> 4) << 24);
            for (u32 t = pair; ok && t < tiles; t += pairs, ++turn_acc) {
                if (turn_acc && !wait_one(&sh, &sh.acc_empty, (turn_acc - 1) & 1, g)) { ok = false; break; }
                tm_fence_after();
                for (u32 k = 0; k < g.col_tiles; ++k, ++step) {
                    const u32 s = step % STAGES, parity = (step / STAGES) & 1;
                    if (!wait_one(&sh, &sh.ready[s], parity, g)) { ok = false; break; }
                    tm_fence_after();
                    const u32 st = base + s * STAGE;
                    const u32 sa = tmem + SPAN + s * SF_COLS, sb = sa + PIECES * 4;
                    const u64 da = desc_swizzled(st), db = desc_swizzled(st + CODES);
#pragma unroll
                    for (u32 i = 0; i < 4; ++i) {  // 64 columns = 32 bytes of codes each
                        if (FMT == MX4_E4M3_16) {
                            tm2_mma_block16(tmem, da + 2 * i, db + 2 * i, IDESC, sa + i * 4, sb + i * 8, k || i);
                        } else {
                            const u32 half = (i & 1) * 2, j = i >> 1;      // a piece serves two instructions
                            tm2_mma_block32(tmem, da + 2 * i, db + 2 * i, IDESC | (half << 4) | (half << 29), sa + j * 4, sb + j * 8, k || i);
                        }
                    }
                    tm2_commit(&sh.empty[s]);
                }
                if (ok) tm2_commit(&sh.acc_full);
            }
            if (!ok) {                             // what has been issued is done before tensor memory goes
                tm2_commit(&sh.acc_full);
                drain_one(&sh.acc_full, turn_acc & 1);
            }
        }
    } else if (warp >= STORE_WARPS + 2) {
        // Scales from shared memory to the tensor-memory lanes of the warp's place: row 32 c + l of a piece is four bytes of
        // lane l, column c.  (The tensor core's own copy instruction queues up with the products, 65 cycles for 512 bytes.)
        const u32 quarter = warp & 3;
        u32 step = 0;
        bool ok = true;
        for (u32 t = pair; ok && t < tiles; t += pairs) {
            for (u32 k = 0; k < g.col_tiles; ++k, ++step) {
                const u32 s = step % STAGES;
                const bool landed = lane == 0 ? wait_one(&sh, &sh.full[s], (step / STAGES) & 1, g) : true;
                if (!__all_sync(0xffffffffu, landed)) { ok = false; break; }
                const uint4* from = reinterpret_cast<const uint4*>(smem + s * STAGE + 2 * CODES) + lane;
                // each stage has scale columns of its own, free again when the stage is
                const u32 sa = tmem + ((quarter * 32) << 16) + SPAN + s * SF_COLS, sb = sa + PIECES * 4;
                uint4 a[PIECES], b[PIECES * 2];
#pragma unroll
                for (u32 j = 0; j < PIECES; ++j) {
                    a[j] = from[j * 32];
                    b[2 * j] = from[(PIECES + j) * 32];
                    b[2 * j + 1] = from[(2 * PIECES + j) * 32];
                }
                if (FMT == MX4_E4M3_16) {
                    tm_store16(sa, reinterpret_cast<const u32*>(a));
                    tm_store32(sb, reinterpret_cast<const u32*>(b));
                } else {
                    tm_store8(sa, reinterpret_cast<const u32*>(a));
                    tm_store16(sb, reinterpret_cast<const u32*>(b));
                }
                tm_wait_store();
                tm_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(cluster_address(&sh.ready[s], 0));
            }
        }
    } else if (warp < STORE_WARPS) {
        const float alpha = (g.m.scale ? __ldg(g.m.scale) : 1.f) * (g.n.scale ? __ldg(g.n.scale) : 1.f);
        const u32 quarter = warp & 3, c0 = (warp >> 2) * 128;              // a warp reads the tensor-memory lanes of its place
        u32 turn = 0;
        for (u32 t = pair; t < tiles; t += pairs, ++turn) {
            u32 mt, nt;
            place(g, t, mt, nt);
            __syncwarp();
            const bool ready = lane == 0 ? wait_one(&sh, &sh.acc_full, turn & 1, g) : true;
            if (!__all_sync(0xffffffffu, ready)) break;
            tm_fence_after();
            const u64 m = (u64)(2 * mt + rank) * MX4_ROWS + quarter * 32 + lane;
            const u64 n0 = (u64)nt * SPAN + c0;
            const u32 cols = n0 < g.n.rows ? (u32)min((u64)128, g.n.rows - n0) : 0u;
            T* y = static_cast<T*>(g.y) + m * g.stride + n0;
            // 16-bit results wait in registers until the accumulator has been handed back; fp32 ones, twice as many, leave in
            // four parts, the last one after that
            constexpr u32 PER = 4 / sizeof(T), HELD = sizeof(T) == 2 ? 64 : 32;      // results in a word; words in registers
            u32 w[HELD];
#pragma unroll
            for (u32 c = 0; c < 128; c += 32) {
                u32 v[32];
                tm_load32(tmem + ((quarter * 32) << 16) + c0 + c, v);
                tm_wait_load();
                if (c == 96) {                     // all columns are in registers
                    tm_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(cluster_address(&sh.acc_empty, 0));
                }
#pragma unroll
                for (u32 i = 0; i < 32; i += PER) {
                    float f[PER];
#pragma unroll
                    for (u32 e = 0; e < PER; ++e) {
                        f[e] = __uint_as_float(v[i + e]) * alpha;
                        if (g.bias && c + i + e < cols) f[e] += __ldg(g.bias + n0 + c + i + e);
                    }
                    if constexpr (PER == 2) w[(c + i) / 2] = two<DT>(f[0], f[1]);
                    else w[i] = __float_as_uint(f[0]);
                }
                if (PER == 1 && m < g.m.rows) put_row<T, HELD>(y + c, w, cols > c ? cols - c : 0, g.wide_store);
            }
            if (PER == 2 && m < g.m.rows) put_row<T, HELD>(y, w, cols, g.wide_store);
        }
    }
    __syncwarp();
    tm_fence_before();
    __syncthreads();
    cluster_barrier();                             // neither CTA's memory is needed any more
    if (warp == STORE_WARPS + 1) tm2_dealloc(tmem, TMEM_COLS);
}

template <int FMT, int DT>
bool launch_as(int sms, cudaStream_t s, const WideArgs& g) {
    const u32 smem = stage_bytes<FMT>() * stages<FMT>() + 1024;
    if (cudaFuncSetAttribute(wide_kernel<FMT, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
    const u64 tiles = (u64)g.m_tiles * g.n_tiles;
    const u32 pairs = (u32)(tiles < (u64)(sms / 2) ? tiles : (u64)(sms / 2));
    wide_kernel<FMT, DT><<<pairs * 2, THREADS, smem, s>>>(g);
    return true;
}

}  // namespace

bool launch_mx4_matmul_wide(int sms, cudaStream_t s, const Mx4Operand& a, const Mx4Operand& b, u64 cols, int fmt,
                            const Mx4Result& r, u64 wait_ns, u32* flag) {
    WideArgs g{};
    g.m = a;
    g.n = b;
    g.col_tiles = mx4_col_tiles(cols);
    g.m_tiles = (u32)((a.rows + SPAN - 1) / SPAN);
    g.n_tiles = (u32)((b.rows + SPAN - 1) / SPAN);
    g.y = r.y;
    g.stride = r.stride;
    g.bias = r.bias;
    const u64 size = r.dtype == DT_F32 ? 4 : 2;
    g.wide_store = ((reinterpret_cast<uintptr_t>(r.y) | (r.stride * size)) & 31) == 0;
    g.wait_ns = wait_ns;
    g.flag = flag;
#define EXCP_MM(DT) (fmt == MX4_E4M3_16 ? launch_as<MX4_E4M3_16, DT>(sms, s, g) : launch_as<MX4_E8M0_32, DT>(sms, s, g))
    return r.dtype == DT_F32 ? EXCP_MM(DT_F32) : r.dtype == DT_F16 ? EXCP_MM(DT_F16) : EXCP_MM(DT_BF16);
#undef EXCP_MM
}

}  // namespace excp
