// Product of two microscaled 4-bit matrices, many rows on both sides (see mx4_matmul.cu for few).
//
// Bound: the tensor cores (a 256 x 256 x 64 step measures about 200 cycles), and close behind them shared memory: 4-bit
// operands run through the matrix pipe so fast that a CTA alone would write and read 200 bytes of tiles per cycle.  A pair of
// CTAs therefore works on one 256 x 256 tile (tcgen05 cta_group::2): each holds 128 rows of a and half the rows of b, which takes
// a third off the traffic.  4096 x 4096 x 32000: blocks of 16 220 us (4.9 PFLOP/s), blocks of 32 204 us (5.3); 4096 x 16384 x 8192
// 192 us (5.7); back to back at the power cap (1.41 GHz) 247 us.  A library product of the same formats took 203 us, and 230 back
// to back.  3.5 % of the first case is its last turn: 2000 tiles on 74 pairs are 27 full turns and two tiles.
//
// Persistent pairs: pair p computes tiles p, p + pairs, ...  Roles in each CTA: warps 0..7 write the result, warps 8..11
// bring the block scales to tensor memory, warps 12..14 fetch (contiguous bulk copies, the packed layout is the tensor
// core's), warp 15 of the even CTA issues the matrix instructions.  The accumulator (256 columns of tensor memory) is read
// into registers in one go and handed back before it is converted and written, so that the next tile waits for a
// few hundred cycles only.
// Every wait for a copy, a product or another warp is bounded; where one runs out the CTA raises the handle's flag, lets its copies land and
// leaves (the partner's waits run out in turn).  The two that hardware gives no limit, for tensor memory and at the pair's barrier,
// depend only on CTAs whose own waits are bounded.
#include "mx4_pipe.cuh"

namespace excp {
namespace {

constexpr int STORE_WARPS = 8;
constexpr int SCALE_WARPS = 4;
constexpr int FETCH_WARPS = 3;
constexpr u32 SCALE_WARP = STORE_WARPS, FETCH_WARP = SCALE_WARP + SCALE_WARPS, PRODUCT_WARP = FETCH_WARP + FETCH_WARPS;
constexpr int THREADS = (PRODUCT_WARP + 1) * 32;
constexpr int UP = 168, DOWN = 88;                 // registers per thread of the store warps and of the others
constexpr u32 CODES = MX4_ROWS * 128;              // codes of one operand tile
constexpr u32 SPAN = 2 * MX4_ROWS;                 // rows of a and of b per pair
// Tiles of m that are visited before the next tile of n.  Under the power cap what the tiles are fetched with counts:
// 4096 x 4096 x 32000 back to back 282, 265, 253, 247 us with 2, 4, 8, 16.
constexpr u32 GROUP = 16;

template <int FMT> __host__ __device__ constexpr int stages() { return FMT == MX4_E4M3_16 ? 5 : 6; }
// A stage: tile of m (codes, scales), own tile of n (codes, scales), scales of the partner's tile of n.
template <int FMT> __host__ __device__ constexpr u32 stage_bytes() { return 2 * CODES + 3 * mx4_scale_bytes(FMT); }

struct WideArgs {
    Mx4Operand m, n;                               // on the M side (TMEM lanes) and the N side (columns)
    u32 col_tiles, m_tiles, n_tiles;
    void* y;
    u64 stride;
    const float* bias;                             // per row of b
    // Usually a is m: a lane has a row of y and writes 32 bytes at a time.  Where rows of y do not start on 32 bytes the operands
    // change places: a lane has a column, and neighbouring lanes write neighbouring results.
    u32 turned;
    u32 early;                                     // the launch before packs a, and b may be fetched before it ends
    u64 wait_ns;
    u32* flag;
};

template <int FMT>
struct Shared {
    unsigned long long full[stages<FMT>()];        // own copies have landed
    unsigned long long ready[stages<FMT>()];       // even CTA: both CTAs' have, and the scales are in tensor memory
    unsigned long long empty[stages<FMT>()];       // the stage has been multiplied
    unsigned long long acc_full, acc_empty;
    unsigned long long last;                       // everything that was issued is done; one turn only
    u32 tmem;
    volatile u32 abort;
};

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
__device__ __forceinline__ void put_row(T* y, const u32 (&w)[WORDS], u32 cols) {
    constexpr u32 PER = 4 / sizeof(T);
#pragma unroll
    for (u32 i = 0; i < WORDS; i += 8) {
        if ((i + 8) * PER <= cols) {
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
    const u32 warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const u32 rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const u32 tiles = g.m_tiles * g.n_tiles;

    if (!g.early) wait_for_previous();
    let_next_start();
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&sh.full[s], FETCH_WARPS); mbar_init(&sh.ready[s], 2 * SCALE_WARPS); mbar_init(&sh.empty[s], 1); }
        mbar_init(&sh.acc_full, 1);
        mbar_init(&sh.last, 1);
        mbar_init(&sh.acc_empty, 2 * STORE_WARPS);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == PRODUCT_WARP) tm2_alloc(&sh.tmem, TMEM_COLS);
    tm_fence_before();
    __syncthreads();
    cluster_barrier();                             // the partner's barriers are ready
    tm_fence_after();
    const u32 tmem = sh.tmem;

    // The store warps hold 128 accumulator columns at a time: they take the registers that the others do without.
    static_assert(THREADS == 512 && STORE_WARPS == 8 && 256 * UP + 256 * DOWN <= 512 * 128, "registers: launched with 128 a thread");

    if (warp >= FETCH_WARP) {
        registers_down<DOWN>();
        if (warp < PRODUCT_WARP) {
            // Three warps fetch: the tile of m, the own tile of n, and of the partner's tile of n the scales (each CTA's tensor memory
            // holds those of all of n's rows).  Issuing a copy takes one or two hundred cycles, more than a stage has for three.
            const u32 item = warp - FETCH_WARP;
            Ring<STAGES> ring;
            u32 filled = 0;
            bool ok = true;
            if (g.early && (item == 0) != (g.turned != 0)) wait_for_previous();    // only a depends on the launch before
            for (u32 t = pair; ok && t < tiles; t += pairs) {
                u32 mt, nt;
                place(g, t, mt, nt);
                const u64 rows = item == 0 ? g.m.rows : g.n.rows;
                const u32 rt = item == 0 ? 2 * mt + rank : 2 * nt + (item == 1 ? rank : 1 - rank);
                // row tiles past the end are not fetched: their rows' results are not written
                const bool there = (u64)rt * MX4_ROWS < rows;
                const u32 height = there ? mx4_tile_height(rows, rt) : 0, advance = height * 128 + SB;
                const unsigned char* from = (item == 0 ? g.m.p : g.n.p) + (there ? mx4_tile_offset(rows, g.col_tiles, FMT, rt, 0) : 0);
                const u32 at = item == 0 ? 0 : item == 1 ? CODES + SB : 2 * (CODES + SB);
                // codes at their place and the scales, which follow them in the packed tile, behind 128 rows: a full tile is one copy
                const bool full = there && height == MX4_ROWS && item != 2;
                for (u32 k = 0; k < g.col_tiles; ++k) {
                    if (filled >= STAGES && !wait_warp(&sh, &sh.empty[ring.s], ring.parity ^ 1, g.wait_ns, g.flag)) { ok = false; break; }
                    unsigned char* to = smem + ring.s * STAGE + at;
                    unsigned long long* bar = &sh.full[ring.s];
                    if (elect_one()) {
                        mbar_arrive_expect_tx(bar, !there ? 0 : item == 2 ? SB : advance);
                        if (full) {
                            bulk_g2s(to, from, CODES + SB, bar);
                        } else if (there) {
                            if (item != 2) bulk_g2s(to, from, height * 128, bar);
                            bulk_g2s(item == 2 ? to : to + CODES, from + height * 128, SB, bar);
                        }
                    }
                    __syncwarp();
                    from += advance;
                    ++filled;
                    ring.next();
                }
            }
            // no copy may be in flight when the CTA leaves: the last turn of every stage that was filled
            for (u32 i = 0; i < STAGES && i < filled; ++i) {
                if (ring.s == 0) { ring.s = STAGES; ring.parity ^= 1; }
                --ring.s;
                drain_warp(&sh.full[ring.s], ring.parity);
            }
        } else if (rank == 0) {
            constexpr u32 IDESC = (1u << 7) | (1u << 10) | ((SPAN >> 3) << 17) | (FMT == MX4_E8M0_32 ? 1u << 23 : 0u) | ((SPAN >> 4) << 24);
            Ring<STAGES> ring;
            u32 turn = 0;
            bool ok = true;
            for (u32 t = pair; ok && t < tiles; t += pairs, ++turn) {
                if (turn && !wait_warp(&sh, &sh.acc_empty, (turn - 1) & 1, g.wait_ns, g.flag)) { ok = false; break; }
                for (u32 k = 0; k < g.col_tiles; ++k) {
                    if (!wait_warp(&sh, &sh.ready[ring.s], ring.parity, g.wait_ns, g.flag)) { ok = false; break; }
                    tm_fence_after();
                    const u32 st = base + ring.s * STAGE;
                    const u32 sa = tmem + SPAN + ring.s * SF_COLS, sb = sa + PIECES * 4;
                    const u64 da = desc_swizzled(st), db = desc_swizzled(st + CODES + SB);
                    if (elect_one()) {
#pragma unroll
                        for (u32 i = 0; i < 4; ++i) {  // 64 columns = 32 bytes of codes each
                            if (FMT == MX4_E4M3_16) {
                                tm2_mma_block16(tmem, da + 2 * i, db + 2 * i, IDESC, sa + i * 4, sb + i * 8, k || i);
                            } else {
                                const u32 half = (i & 1) * 2, j = i >> 1;      // a piece serves two instructions
                                tm2_mma_block32(tmem, da + 2 * i, db + 2 * i, IDESC | (half << 4) | (half << 29), sa + j * 4, sb + j * 8, k || i);
                            }
                        }
                        tm2_commit(&sh.empty[ring.s]);
                        if (k + 1 == g.col_tiles) tm2_commit(&sh.acc_full);
                    }
                    __syncwarp();
                    ring.next();
                }
            }
            if (elect_one()) tm2_commit(&sh.last);
            __syncwarp();
        }
    } else if (warp >= SCALE_WARP) {
        registers_down<DOWN>();
        // Scales from shared memory to the tensor-memory lanes of the warp's place: row 32 c + l of a piece is four bytes of
        // lane l, column c.  (The tensor core's own copy instruction queues up with the products, 65 cycles for 512 bytes.)
        const u32 quarter = warp & 3;
        Ring<STAGES> ring;
        bool ok = true;
        for (u32 t = pair; ok && t < tiles; t += pairs) {
            for (u32 k = 0; k < g.col_tiles; ++k) {
                if (!wait_warp(&sh, &sh.full[ring.s], ring.parity, g.wait_ns, g.flag)) { ok = false; break; }
                const uint4* from = reinterpret_cast<const uint4*>(smem + ring.s * STAGE + CODES) + lane;
                const uint4* own = from + (CODES + SB) / 16;
                const uint4* other = own + SB / 16;
                const uint4* n0 = rank == 0 ? own : other;
                const uint4* n1 = rank == 0 ? other : own;
                // each stage has scale columns of its own, free again when the stage is
                const u32 sa = tmem + ((quarter * 32) << 16) + SPAN + ring.s * SF_COLS, sb = sa + PIECES * 4;
                uint4 a[PIECES], b[PIECES * 2];
#pragma unroll
                for (u32 j = 0; j < PIECES; ++j) {
                    a[j] = from[j * 32];
                    b[2 * j] = n0[j * 32];
                    b[2 * j + 1] = n1[j * 32];
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
                if (elect_one()) mbar_arrive_cluster(cluster_address(&sh.ready[ring.s], 0));
                ring.next();
            }
        }
    } else {
        registers_up<UP>();
        const TensorScales by = tensor_scales(g.m.scale, g.n.scale);
        const u32 quarter = warp & 3, c0 = (warp >> 2) * 128;              // a warp reads the tensor-memory lanes of its place
        u32 turn = 0;
        for (u32 t = pair; t < tiles; t += pairs, ++turn) {
            u32 mt, nt;
            place(g, t, mt, nt);
            __syncwarp();
            if (!wait_warp(&sh, &sh.acc_full, turn & 1, g.wait_ns, g.flag)) break;
            tm_fence_after();
            const u64 m = (u64)(2 * mt + rank) * MX4_ROWS + quarter * 32 + lane;
            const u64 n0 = (u64)nt * SPAN + c0;
            const u32 cols = n0 < g.n.rows ? (u32)min((u64)128, g.n.rows - n0) : 0u;
            const u32 from = tmem + ((quarter * 32) << 16) + c0;
            u32 v[128];
#pragma unroll
            for (u32 i = 0; i < 4; ++i) tm_load32(from + i * 32, v + i * 32);
            tm_wait_load();
            tm_fence_before();
            __syncwarp();
            if (elect_one()) mbar_arrive_cluster(cluster_address(&sh.acc_empty, 0));

            constexpr u32 PART = 32, PER = 4 / sizeof(T);                  // columns at a time; results in a word
            if (g.turned) {
                T* const y = static_cast<T*>(g.y) + n0 * g.stride + m;
                const float bias = g.bias && m < g.m.rows ? __ldg(g.bias + m) : 0.f;
#pragma unroll
                for (u32 p = 0; p < 128; p += PART) {
                    float f[PART];
#pragma unroll
                    for (u32 i = 0; i < PART; ++i) f[i] = __uint_as_float(v[p + i]) * by.first;
                    if (by.second != 1.f) {
#pragma unroll
                        for (u32 i = 0; i < PART; ++i) f[i] *= by.second;
                    }
                    if (g.bias) {
#pragma unroll
                        for (u32 i = 0; i < PART; ++i) f[i] += bias;
                    }
                    if (m >= g.m.rows) continue;
                    if (p + PART <= cols) {
#pragma unroll
                        for (u32 i = 0; i < PART; ++i) wput(y + (p + i) * g.stride, 0, f[i]);
                    } else {
#pragma unroll
                        for (u32 i = 0; i < PART; ++i) if (p + i < cols) wput(y + (p + i) * g.stride, 0, f[i]);
                    }
                }
                continue;
            }
            T* const y = static_cast<T*>(g.y) + m * g.stride + n0;
#pragma unroll
            for (u32 p = 0; p < 128; p += PART) {
                float f[PART];
#pragma unroll
                for (u32 i = 0; i < PART; ++i) f[i] = __uint_as_float(v[p + i]) * by.first;
                if (by.second != 1.f) {
#pragma unroll
                    for (u32 i = 0; i < PART; ++i) f[i] *= by.second;
                }
                if (g.bias) {
#pragma unroll
                    for (u32 i = 0; i < PART; ++i) f[i] += p + i < cols ? __ldg(g.bias + n0 + p + i) : 0.f;
                }
                u32 w[PART / PER];
#pragma unroll
                for (u32 i = 0; i < PART; i += PER) {
                    if constexpr (PER == 2) w[i / 2] = two<DT>(f[i], f[i + 1]);
                    else w[i] = __float_as_uint(f[i]);
                }
                if (m < g.m.rows) put_row<T, PART / PER>(y + p, w, cols > p ? cols - p : 0);
            }
        }
    }
    __syncwarp();
    tm_fence_before();
    __syncthreads();
    // What has been issued is done before tensor memory and the CTAs go, also where only the warps that wait for it gave up.
    // (acc_full cannot say so: while a tile is unfinished, a wait for the next one is met by the one before it.)
    if (warp == PRODUCT_WARP) drain_warp(&sh.last, 0);
    cluster_barrier();                             // neither CTA's memory is needed any more
    if (warp == PRODUCT_WARP) tm2_dealloc(tmem, TMEM_COLS);
}

template <int FMT, int DT>
bool launch_as(int sms, cudaStream_t s, const WideArgs& g) {
    const u32 smem = stage_bytes<FMT>() * stages<FMT>() + 1024;
    static std::atomic<u64> allowed{0};
    if (!allow_smem(wide_kernel<FMT, DT>, allowed, smem)) return false;
    const u64 tiles = (u64)g.m_tiles * g.n_tiles;
    const u32 pairs = (u32)(tiles < (u64)(sms / 2) ? tiles : (u64)(sms / 2));
    return launch_chained(wide_kernel<FMT, DT>, pairs * 2, THREADS, smem, 0, s, g);
}

}  // namespace

bool launch_mx4_matmul_wide(int sms, cudaStream_t s, const Mx4Operand& a, const Mx4Operand& b, u64 cols, int fmt,
                            const Mx4Result& r, u64 wait_ns, u32* flag, bool behind) {
    WideArgs g{};
    const u64 size = r.dtype == DT_F32 ? 4 : 2;
    g.turned = ((reinterpret_cast<uintptr_t>(r.y) | (r.stride * size)) & 31) != 0;
    g.m = g.turned ? b : a;
    g.n = g.turned ? a : b;
    g.col_tiles = mx4_col_tiles(cols);
    g.m_tiles = (u32)((g.m.rows + SPAN - 1) / SPAN);
    g.n_tiles = (u32)((g.n.rows + SPAN - 1) / SPAN);
    g.y = r.y;
    g.stride = r.stride;
    g.bias = r.bias;
    g.early = behind;
    g.wait_ns = wait_ns;
    g.flag = flag;
#define EXCP_MM(DT) (fmt == MX4_E4M3_16 ? launch_as<MX4_E4M3_16, DT>(sms, s, g) : launch_as<MX4_E8M0_32, DT>(sms, s, g))
    return r.dtype == DT_F32 ? EXCP_MM(DT_F32) : r.dtype == DT_F16 ? EXCP_MM(DT_F16) : EXCP_MM(DT_BF16);
#undef EXCP_MM
}

}  // namespace excp
