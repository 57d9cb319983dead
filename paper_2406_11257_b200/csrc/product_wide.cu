// The product with plain 16-bit operands, many rows on both sides (product.cu: few).
//
// Bound: the tensor cores, and soon the power cap.  4096 x 4096 x 11008 bf16: 232 us in a burst (1.6 PFLOP/s; a library product on the
// same card 238), dx 255 (236), dw to 32 bits 256; back to back the clock falls to 1.4 GHz, and with it all of them to some 300.
// A pair of CTAs works on a tile of 256 x 256 (tcgen05 cta_group::2): each holds 128 rows of the M side and
// half of the N side's 256, so that a step of 64 columns costs a CTA 32 KB of shared memory for 512 cycles of products.  The
// accumulators of two tiles fit tensor memory: one is written out while the next is summed.
//
// Persistent pairs: pair p computes tiles p, p + pairs, ...  Roles in each CTA: warps 0..7 write the result, warps 8 to 11 fetch the
// two operands (tensor maps; what lies past an edge comes as 0), warp 12 of the even CTA issues the products, and that of the odd
// CTA tells it of its own copies' landing.
// Every wait for a copy, a product or another warp is bounded; where one runs out the CTA raises the handle's flag, lets its copies land and
// leaves (the partner's waits run out in turn).  The two that hardware gives no limit, for tensor memory and at the pair's barrier,
// depend only on CTAs whose own waits are bounded.
#include "product.cuh"

namespace excp {
namespace {

constexpr int STORE_WARPS = 8;
constexpr u32 FETCH_WARPS = 2;                     // per operand, every other stage
constexpr u32 FETCH_WARP = STORE_WARPS, PRODUCT_WARP = FETCH_WARP + 2 * FETCH_WARPS;
// Where sums are taken in runs the store warps hold the sum of the runs, 128 columns a thread: they take the registers that the others (and
// three warps that do nothing) do without.
template <bool RUNS> __host__ __device__ constexpr int threads() { return RUNS ? 512 : (int)(PRODUCT_WARP + 1) * 32; }
constexpr int UP = 200, DOWN = 56;                 // registers a thread, of 128 at launch
static_assert(256 * UP + 256 * DOWN <= 512 * 128, "registers");
constexpr int STAGES = 6;
constexpr u32 SPAN = 2 * PR_TILE;                  // rows of m and of n per pair
constexpr u32 HALF = PR_TILE * PR_K * 2, STAGE = 2 * HALF;
constexpr u32 OUT_BYTES = 4096;                    // of a warp's results on their way out
constexpr u32 SMEM = STAGES * STAGE + STORE_WARPS * OUT_BYTES + 1024;        // no other CTA that uses tensor memory fits beside it (product.cu: why that matters)
constexpr u32 GROUP = 16;                          // tiles of m that are visited before the next tile of n

struct WideArgs {
    CUtensorMap m, n;                              // on the M side (lanes of tensor memory) and the N side (columns)
    CUtensorMap y;                                 // not where they change places
    u32 m_along_k, n_along_k, bf16;
    u32 k_tiles, m_tiles, n_tiles;
    u32 run;                                       // stages
    // Usually a is m: a lane has a row of c.  Where rows of y do not start on 16 bytes the operands change places: a lane has a column,
    // and neighbouring lanes write neighbouring results.
    u32 turned;
    EndArgs end;
    u64 wait_ns;
    u32* flag;
};

struct Shared {
    unsigned long long full[STAGES];               // own copies have landed
    unsigned long long peer[STAGES];               // even CTA: the partner's have
    unsigned long long empty[STAGES];              // the stage has been multiplied
    unsigned long long acc_full[2], acc_empty[2];
    unsigned long long last;                       // everything that was issued is done; one turn only
    u32 tmem;
    volatile u32 abort;
};

__device__ __forceinline__ void place(const WideArgs& g, u32 t, u32& mt, u32& nt) {
    const u32 per_group = GROUP * g.n_tiles;
    const u32 group = t / per_group, inside = t - group * per_group;
    const u32 rows = min(GROUP, g.m_tiles - group * GROUP);
    nt = inside / rows;
    mt = group * GROUP + inside - nt * rows;
}

template <int DT, bool RUNS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(threads<RUNS>(), 1) wide_product_kernel(const __grid_constant__ WideArgs g) {
    constexpr u32 TMEM_COLS = 512;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared sh;
    // the swizzle goes by address: stages start on 1024 bytes (the same offset in both CTAs)
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const u32 base = smem_u32(smem);
    const u32 warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const u32 rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const u32 tiles = g.m_tiles * g.n_tiles;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&sh.full[s], 2); mbar_init(&sh.peer[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh.acc_full[b], 1); mbar_init(&sh.acc_empty[b], 2 * STORE_WARPS); }
        mbar_init(&sh.last, 1);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == PRODUCT_WARP) tm2_alloc(&sh.tmem, TMEM_COLS);
    if (warp == FETCH_WARP && elect_one()) { tma_prefetch_map(&g.m); tma_prefetch_map(&g.n); }
    __syncwarp();
    wait_for_previous();
    let_next_start();
    tm_fence_before();
    __syncthreads();
    cluster_barrier();                             // the partner's barriers are ready
    tm_fence_after();
    const u32 tmem = sh.tmem;
    // stages that are added up in one accumulator
    const u32 run = RUNS ? g.run : g.k_tiles;
    if (warp >= FETCH_WARP && warp < PRODUCT_WARP) {
        if constexpr (RUNS) registers_down<DOWN>();
        const bool is_n = warp >= FETCH_WARP + FETCH_WARPS;
        const CUtensorMap* map = is_n ? &g.n : &g.m;
        const bool along_k = is_n ? g.n_along_k : g.m_along_k;
        const u32 mine = (warp - FETCH_WARP) % FETCH_WARPS;
        Ring<STAGES> ring;
        u32 filled = 0;                            // stages so far, the other warps' among them
        bool ok = true;
        for (u32 t = pair; ok && t < tiles; t += pairs) {
            u32 mt, nt;
            place(g, t, mt, nt);
            const u32 row = ((is_n ? nt : mt) * 2 + rank) * PR_TILE;
            for (u32 k = 0; k < g.k_tiles; ++k, ++filled, ring.next()) {
                if (filled % FETCH_WARPS != mine) continue;
                if (filled >= STAGES && !wait_warp(&sh, &sh.empty[ring.s], ring.parity ^ 1, g.wait_ns, g.flag)) { ok = false; break; }
                unsigned char* to = smem + ring.s * STAGE + (is_n ? HALF : 0);
                unsigned long long* bar = &sh.full[ring.s];
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar, HALF);
                    if (along_k) {
                        tma_load_2d(to, map, k * PR_K, row, bar);
                    } else {
                        tma_load_2d(to, map, row, k * PR_K, bar);
                        tma_load_2d(to + PR_CHUNK_BYTES, map, row + PR_CHUNK, k * PR_K, bar);
                    }
                }
                __syncwarp();
            }
        }
        // no copy may be in flight when the CTA leaves: the last turn of every stage that was filled
        for (u32 i = 0; i < STAGES && i < filled; ++i) {
            if (ring.s == 0) { ring.s = STAGES; ring.parity ^= 1; }
            --ring.s;
            drain_warp(&sh.full[ring.s], ring.parity);
        }
    } else if (warp >= PRODUCT_WARP) {
        if constexpr (RUNS) registers_down<DOWN>();
        if (warp > PRODUCT_WARP) {                 // nothing
        } else if (rank == 0) {
            const u32 idesc = product_idesc(g.bf16, g.m_along_k, g.n_along_k, SPAN, SPAN);
            const u32 step_m = product_desc_step(g.m_along_k), step_n = product_desc_step(g.n_along_k);
            Ring<STAGES> ring;
            u32 turn = 0;
            bool ok = true;
            for (u32 t = pair; ok && t < tiles; t += pairs) {
                u32 b = 0, left = 0;                   // the accumulator, stages that it still takes
                for (u32 k = 0; k < g.k_tiles; ++k) {
                    const bool first = left == 0;
                    if (first) {
                        b = turn & 1;
                        left = min(run, g.k_tiles - k);
                        if (turn >= 2 && !wait_warp(&sh, &sh.acc_empty[b], ((turn >> 1) - 1) & 1, g.wait_ns, g.flag)) { ok = false; break; }
                        tm_fence_after();
                        ++turn;
                    }
                    if (!wait_warp(&sh, &sh.full[ring.s], ring.parity, g.wait_ns, g.flag) ||
                        !wait_warp(&sh, &sh.peer[ring.s], ring.parity, g.wait_ns, g.flag)) { ok = false; break; }
                    const u32 st = base + ring.s * STAGE, acc = tmem + b * SPAN;
                    const u64 dm = product_desc(st, g.m_along_k), dn = product_desc(st + HALF, g.n_along_k);
                    --left;
                    if (elect_one()) {
#pragma unroll
                        for (u32 i = 0; i < PR_K / 16; ++i) tm2_mma_f16(acc, dm + i * step_m, dn + i * step_n, idesc, !first || i);
                        tm2_commit(&sh.empty[ring.s]);
                        if (left == 0) tm2_commit(&sh.acc_full[b]);
                    }
                    __syncwarp();
                    ring.next();
                }
            }
            if (elect_one()) tm2_commit(&sh.last);
            __syncwarp();
        } else {
            Ring<STAGES> ring;
            bool ok = true;
            for (u32 t = pair; ok && t < tiles; t += pairs) {
                for (u32 k = 0; k < g.k_tiles; ++k) {
                    if (!wait_warp(&sh, &sh.full[ring.s], ring.parity, g.wait_ns, g.flag)) { ok = false; break; }
                    if (elect_one()) mbar_arrive_cluster(cluster_address(&sh.peer[ring.s], 0));
                    __syncwarp();
                    ring.next();
                }
            }
        }
    } else {
        if constexpr (RUNS) registers_up<UP>();
        const u32 quarter = warp & 3, c0 = (warp >> 2) * PR_TILE;          // a warp reads the tensor-memory lanes of its place
        const u32 lanes = tmem + ((quarter * 32) << 16) + c0;
        const u64 n_rows = g.turned ? g.end.rows : g.end.cols;
        u32 out = 0;
        auto put = [&](u64 m, u64 n, float bias, float (&f)[32]) {         // 32 neighbouring columns of the accumulator
            if (n >= n_rows) return;
            if (g.turned) end_column<DT, 32>(g.end, n, m, (u32)min((u64)32, n_rows - n), bias, f);
            else end_rows<DT, OUT_BYTES>(g.end, &g.y, smem + STAGES * STAGE + warp * OUT_BYTES, out, m, n, f);
        };
        auto release = [&](u32 b) {                // the accumulator is free again
            tm_fence_before();
            __syncwarp();
            if (elect_one()) mbar_arrive_cluster(cluster_address(&sh.acc_empty[b], 0));
            __syncwarp();
        };
        u32 turn = 0;
        bool ok = true;
        for (u32 t = pair; ok && t < tiles; t += pairs) {
            u32 mt, nt;
            place(g, t, mt, nt);
            const u64 m = (u64)(2 * mt + rank) * PR_TILE + quarter * 32 + lane, n0 = (u64)nt * SPAN + c0;
            const float bias = g.turned ? column_bias(g.end, m) : 0.f;
            if constexpr (RUNS) {
                float sum[PR_TILE];
#pragma unroll
                for (u32 e = 0; e < PR_TILE; ++e) sum[e] = 0.f;
                for (u32 k = 0; k < g.k_tiles; k += run, ++turn) {
                    const u32 b = turn & 1;
                    __syncwarp();
                    if (!(ok = wait_warp(&sh, &sh.acc_full[b], (turn >> 1) & 1, g.wait_ns, g.flag))) break;
                    tm_fence_after();
#pragma unroll
                    for (u32 p = 0; p < PR_TILE; p += 16) {
                        u32 v[16];
                        tm_load8(lanes + b * SPAN + p, v);
                        tm_load8(lanes + b * SPAN + p + 8, v + 8);
                        tm_wait_load();
#pragma unroll
                        for (u32 e = 0; e < 16; ++e) sum[p + e] += __uint_as_float(v[e]);
                    }
                    release(b);
                }
                if (!ok) break;
                // the sums move up instead of the loop being unrolled: four epilogues are more than the instruction cache holds
#pragma unroll 1
                for (u32 p = 0; p < PR_TILE; p += 32) {
                    float f[32];
#pragma unroll
                    for (u32 e = 0; e < 32; ++e) f[e] = sum[e];
#pragma unroll
                    for (u32 e = 0; e + 32 < PR_TILE; ++e) sum[e] = sum[e + 32];
                    put(m, n0 + p, bias, f);
                }
            } else {
                const u32 b = turn & 1;
                __syncwarp();
                if (!wait_warp(&sh, &sh.acc_full[b], (turn >> 1) & 1, g.wait_ns, g.flag)) break;
                tm_fence_after();
                ++turn;
#pragma unroll 1
                for (u32 p = 0; p < PR_TILE; p += 32) {
                    u32 v[32];
                    __syncwarp();
                    tm_load32(lanes + b * SPAN + p, v);
                    tm_wait_load();
                    if (p + 32 == PR_TILE) release(b);
                    float f[32];
#pragma unroll
                    for (u32 e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]);
                    put(m, n0 + p, bias, f);
                }
            }
        }
        end_rows_done();
    }
    __syncwarp();
    tm_fence_before();
    __syncthreads();
    // What has been issued is done before tensor memory and the CTAs go, also where only the warps that wait for it gave up.
    if (warp == PRODUCT_WARP) drain_warp(&sh.last, 0);
    cluster_barrier();                             // neither CTA's memory is needed any more
    if (warp == PRODUCT_WARP) tm2_dealloc(tmem, TMEM_COLS);
}

template <int DT, bool RUNS>
bool launch_as(int sms, cudaStream_t s, const WideArgs& g) {
    static std::atomic<u64> allowed{0};
    if (!allow_smem(wide_product_kernel<DT, RUNS>, allowed, SMEM)) return false;
    const u64 tiles = (u64)g.m_tiles * g.n_tiles;
    const u32 pairs = (u32)(tiles < (u64)(sms / 2) ? tiles : (u64)(sms / 2));
    return launch_chained(wide_product_kernel<DT, RUNS>, pairs * 2, threads<RUNS>(), SMEM, 0, s, g);
}

}  // namespace

// Measured: a step of 64 columns takes a pair 0.275 us, a tile's epilogue 2 us at 16 bits and some 4 at 32, half of which the last one does
// not hide, and a launch 4.5.
float product_wide_us(const ProductCall& c) {
    const u64 tiles = ((c.a.rows + SPAN - 1) / SPAN) * ((c.b.rows + SPAN - 1) / SPAN), pairs = (u64)(c.sms / 2);
    const float end = c.end.y.dtype == DT_F32 ? 4.f : 2.f, sum = (float)((c.a.k + PR_K - 1) / PR_K) * 0.275f;
    return 4.5f + (float)((tiles + pairs - 1) / pairs) * (sum > end ? sum : end) + 0.5f * end;
}

bool launch_product_wide(cudaStream_t s, const ProductCall& c) {
    WideArgs g;
    g.end = end_args(c.end);
    g.turned = !g.end.y_vec;
    const ProductOperand& m = g.turned ? c.b : c.a;
    const ProductOperand& n = g.turned ? c.a : c.b;
    if (!product_map(&g.m, m, PR_TILE, c.dtype) || !product_map(&g.n, n, PR_TILE, c.dtype)) return false;
    if (!g.turned && !result_map(&g.y, c.end.y)) return false;
    g.m_along_k = m.along_k;
    g.n_along_k = n.along_k;
    g.bf16 = c.dtype == DT_BF16;
    g.k_tiles = (u32)((m.k + PR_K - 1) / PR_K);
    const u32 stages = product_run(c.end) / PR_K, runs = g.k_tiles / stages + (g.k_tiles % stages != 0);
    g.run = (g.k_tiles + runs - 1) / runs;
    g.m_tiles = (u32)((m.rows + SPAN - 1) / SPAN);
    g.n_tiles = (u32)((n.rows + SPAN - 1) / SPAN);
    g.wait_ns = c.wait_ns;
    g.flag = c.flag;
    auto launch = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if constexpr (DT != DT_F32) if (runs == 1) return launch_as<DT, false>(c.sms, s, g);
        return launch_as<DT, true>(c.sms, s, g);
    };
    return c.end.y.dtype == DT_F32 ? launch(std::integral_constant<int, DT_F32>()) : c.end.y.dtype == DT_F16 ? launch(std::integral_constant<int, DT_F16>())
                                                                                                           : launch(std::integral_constant<int, DT_BF16>());
}

}  // namespace excp
