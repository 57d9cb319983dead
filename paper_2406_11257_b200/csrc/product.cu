// The product with plain 16-bit operands: c[i, j] = sum over k of a[i, k] b[j, k], fp32 sums, and its epilogue.
// This file: few rows on one side (the tokens of a decoding step), or too few tiles for the kernel of many (product_wide.cu).
//
// Bound: with few rows the bytes of the larger operand, else what an SM can fetch (about 120 bytes a ns).  The larger operand's rows go on
// the M side of the tensor core (128 per tile), the few rows on the N side, which takes them in steps of 16.  Where there are too few
// tiles for the SMs the columns of a tile are split over a cluster: each CTA sends its part of the accumulator to the CTAs that own its
// columns (bulk copies between their shared memories), which add the parts in a fixed order.
//
// 1 x 4096 -> 11008 bf16 18 us from memory, 16 x 2048 -> 50304 38 us (5.5 TB/s), 333 x 1000 -> 4097 9.9 us, 512 x 1024 -> 1024 6.1 us, one tile
// alone 2.6 us.
//
// Sums are taken in runs of at most PR_RUN columns, whatever the results' types, so that they do not depend on what is done with them.  Up to
// four runs have an accumulator each; of more, all but the last three are added to the first by warps that have nothing else to do, while
// the products go on in the others.  (One run, which loses more the longer it is: 1 x 4096 -> 4096 8.3 us against 8.8, 512 x 4096 -> 4096
// 18.7 against 20.3.)
//
// Roles: warps 0..3 fetch the operands (tensor maps; what lies past an edge comes as 0), warps 4..7 add up runs, warp 8 issues the products, and at
// the end warps 0..7 write the result.
// Every wait for a copy or a product is bounded; where one runs out the CTA raises the handle's flag, lets its copies land and
// leaves.  The two that hardware gives no limit, for tensor memory and at the cluster's barrier, depend only on CTAs whose own
// waits are bounded.
#include "per_device.h"
#include "product.cuh"

namespace excp {
namespace {

constexpr int WORK_WARPS = 8;
constexpr u32 PRODUCT_WARP = WORK_WARPS;
constexpr int THREADS = (PRODUCT_WARP + 1) * 32;
constexpr int BOUND_THREADS = 320;                 // 96 registers a thread: five of the 18 warps of two CTAs share a quarter of the registers
constexpr int STAGES_MAX = 8;
constexpr u32 BOXES_MAX = 2;                       // boxes of 64 columns in a stage
constexpr u32 MAX_SPLIT = 8;
constexpr u32 OUT_BYTES = 8192;                  // of a warp's results on their way out
constexpr u32 ACCS = 4;                            // accumulators at most
constexpr u32 M_BYTES = PR_TILE * PR_K * 2;
constexpr u32 SMEM_MAX = 227 * 1024 - 1024;        // dynamic shared memory of a block, beside what the kernel has of its own
// Tensor memory is given out without a limit on the wait, and a CTA that holds some waits for its cluster: two launches on two streams
// whose CTAs held it from one another would wait for good.  So a CTA takes shared memory in proportion to its columns of tensor memory
// (all of an SM's for 512), and never so little that it fits beside two CTAs of the 4-bit product, which take 256 columns each with 75 KB or
// more: whatever finds room on an SM finds tensor memory.
constexpr u32 SMEM_SM = 228 * 1024, SMEM_LEAST = 76 * 1024;

struct NarrowArgs {
    CUtensorMap m, n, y;                           // y: where lanes have rows and nothing is split
    u32 m_along_k, n_along_k, bf16;
    u32 k_boxes, n_tiles;
    u32 boxes;                                     // of a stage
    u32 nt;                                        // rows of n per CTA: a multiple of 16, at most 256
    u32 n_bytes, stages, tmem_cols;
    u32 accs, runs, run;                           // accumulators, nt columns of tensor memory each; runs of a part's stages, stages of a run
    u32 ring_bytes;                                // of the stages; afterwards the accumulator lies there, or the results on their way out
    u32 per_owner;                                 // columns of the accumulator that a CTA of the cluster joins
    u32 turned;                                    // m is b: a lane has a column of c
    EndArgs end;
    u64 wait_ns;
    u32* flag;
};

struct Shared {
    unsigned long long full[STAGES_MAX];           // copies have landed
    unsigned long long empty[STAGES_MAX];          // the stage has been multiplied
    unsigned long long acc_full[ACCS - 1], acc_empty[ACCS - 1];
    unsigned long long done;
    unsigned long long parts;                      // the other CTAs' parts of the own columns have landed
    u32 tmem;
    volatile u32 abort;
    volatile u32 late;                             // a CTA of the cluster has given up waiting for parts
};

struct Turn {                                      // the place in the ring of stages, and the parity of its current turn
    u32 s = 0, parity = 0;
    __device__ __forceinline__ void next(u32 stages) {
        if (++s == stages) { s = 0; parity ^= 1; }
    }
};

__device__ __forceinline__ void work_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// Shared memory of this CTA -> that of another of the cluster (addresses within the cluster), arriving at a barrier there.
__device__ __forceinline__ void bulk_s2s(u32 to, const void* from, u32 bytes, u32 bar) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(to), "r"(smem_u32(from)), "r"(bytes), "r"(bar) : "memory");
}

template <int DT, bool RUNS>
__global__ void __launch_bounds__(BOUND_THREADS, 2) product_kernel(const __grid_constant__ NarrowArgs g) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared sh;
    const u32 part = cluster_rank(), parts = cluster_size();
    // the swizzle goes by address: stages start on 1024 bytes (the same offset in every CTA)
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const u32 warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const u32 tile = blockIdx.x / parts, mt = tile / g.n_tiles, ntile = tile - mt * g.n_tiles;
    const u32 k_steps = (g.k_boxes + g.boxes - 1) / g.boxes;
    const u32 k0 = (u32)((u64)k_steps * part / parts), k1 = (u32)((u64)k_steps * (part + 1) / parts);
    const u32 box = M_BYTES + g.n_bytes, stage = g.boxes * box;
    // The stages are added up in runs, about equally long.  The first has accumulator 0, the others the rest in turn; those that
    // would find none of their own in the end (`emptied`, from the second on) are added to accumulator 0 on the way.
    const u32 runs = RUNS ? g.runs - (g.runs && k1 - k0 <= (g.runs - 1) * g.run) : k1 > k0;      // a part is one stage shorter than another, or none
    const u32 emptied = RUNS && runs > g.accs ? runs - g.accs : 0;
    const u64 n0 = (u64)ntile * g.nt, n_rows = g.turned ? g.end.rows : g.end.cols;
    const u32 cols = (u32)min((u64)g.nt, n_rows - n0);         // of the accumulator that are results
    // the CTA's own columns of the accumulator, and the others' parts of them: [part][column][row]
    const u32 own = part * g.per_owner, own_cols = own < cols ? min(g.per_owner, cols - own) : 0;
    float* const received = reinterpret_cast<float*>(smem + g.ring_bytes);
    float* const acc = reinterpret_cast<float*>(smem);         // [column][row], once the stages are not needed any more

    if (threadIdx.x == 0) {
        for (u32 s = 0; s < g.stages; ++s) { mbar_init(&sh.full[s], 2 * g.boxes); mbar_init(&sh.empty[s], 1); }
        for (u32 i = 0; i + 1 < ACCS; ++i) { mbar_init(&sh.acc_full[i], 1); mbar_init(&sh.acc_empty[i], 4); }
        mbar_init(&sh.done, 1);
        mbar_init(&sh.parts, 1);
        sh.abort = 0;
        sh.late = 0;
        mbar_fence_init();
        if (parts > 1) mbar_arrive_expect_tx(&sh.parts, (parts - 1) * own_cols * PR_TILE * 4);
    }
    if (warp == PRODUCT_WARP) tm_alloc(&sh.tmem, g.tmem_cols);
    if (warp == 0 && g.k_boxes && elect_one()) { tma_prefetch_map(&g.m); tma_prefetch_map(&g.n); }
    __syncwarp();
    wait_for_previous();
    let_next_start();
    tm_fence_before();
    __syncthreads();
    if (parts > 1) cluster_arrive_release();
    tm_fence_after();
    const u32 tmem = sh.tmem;

    if (warp < 2 * BOXES_MAX) {                    // two warps for each operand, which take turns at its boxes
        const bool is_n = warp >= BOXES_MAX;
        const CUtensorMap* map = is_n ? &g.n : &g.m;
        const bool along_k = is_n ? g.n_along_k : g.m_along_k;
        const u32 first = is_n ? ntile * g.nt : mt * PR_TILE, rows = is_n ? g.nt : PR_TILE, bytes = is_n ? g.n_bytes : M_BYTES;
        u32 turns = k1 - k0;                       // of the ring that are filled
        for (u32 i = warp % BOXES_MAX; i < turns * g.boxes; i += BOXES_MAX) {
            const u32 turn = g.boxes == 1 ? i : i / BOXES_MAX, lap = turn / g.stages, s = turn - lap * g.stages;
            if (lap && !wait_warp(&sh, &sh.empty[s], (lap - 1) & 1, g.wait_ns, g.flag)) { turns = turn; break; }
            unsigned char* to = smem + s * stage + (g.boxes == 1 ? 0 : warp % BOXES_MAX * box) + (is_n ? M_BYTES : 0);
            unsigned long long* bar = &sh.full[s];
            const u32 k = k0 * g.boxes + i, col = k * PR_K;
            if (elect_one()) {
                mbar_arrive_expect_tx(bar, k < g.k_boxes ? bytes : 0);
                if (k < g.k_boxes) {
                    if (along_k) tma_load_2d(to, map, col, first, bar);
                    else for (u32 c = 0; c < rows; c += PR_CHUNK) tma_load_2d(to + c / PR_CHUNK * PR_CHUNK_BYTES, map, first + c, col, bar);
                }
            }
            __syncwarp();
        }
        // no copy may be in flight when the CTA leaves: the last turn of every stage that was filled
        for (u32 t = turns > g.stages ? turns - g.stages : 0; t < turns; ++t) drain_warp(&sh.full[t % g.stages], t / g.stages & 1);
    } else if (warp == PRODUCT_WARP) {
        const u32 idesc = product_idesc(g.bf16, g.m_along_k, g.n_along_k, PR_TILE, g.nt);
        const u32 step_m = product_desc_step(g.m_along_k), step_n = product_desc_step(g.n_along_k);
        Turn ring, acc;
        u32 k = k0, d = tmem;
        bool ok = true;
        for (u32 r = 0; ok && r < runs; ++r) {
            const u32 end = RUNS ? min(k + g.run, k1) : k1;
            if (RUNS && r) {
                if (r > 1) acc.next(g.accs - 1);
                if (r >= g.accs && !(ok = wait_warp(&sh, &sh.acc_empty[acc.s], acc.parity ^ 1, g.wait_ns, g.flag))) break;
                tm_fence_after();
                d = tmem + (1 + acc.s) * g.nt;
            }
            for (u32 begun = 0; k < end; ++k, begun = 1) {
                if (!(ok = wait_warp(&sh, &sh.full[ring.s], ring.parity, g.wait_ns, g.flag))) break;
                const u32 st = smem_u32(smem) + ring.s * stage;
                const u64 dm = product_desc(st, g.m_along_k), dn = product_desc(st + M_BYTES, g.n_along_k);
                if (elect_one()) {
#pragma unroll
                    for (u32 u = 0; u < BOXES_MAX; ++u) {
                        if (u >= g.boxes || k * g.boxes + u >= g.k_boxes) break;
#pragma unroll
                        for (u32 i = 0; i < PR_K / 16; ++i)
                            tm_mma_f16(d, dm + u * (box >> 4) + i * step_m, dn + u * (box >> 4) + i * step_n, idesc, begun | u | i);
                    }
                    tm_commit(&sh.empty[ring.s]);
                }
                __syncwarp();
                ring.next(g.stages);
            }
            if (RUNS && r && r <= emptied) {
                if (elect_one()) tm_commit(&sh.acc_full[acc.s]);
                __syncwarp();
            }
        }
        if (elect_one()) tm_commit(&sh.done);
        __syncwarp();
        drain_warp(&sh.done, 0);                   // what has been issued is done before tensor memory goes
    } else if (RUNS) {                             // warps 4..7, each its place's lanes of tensor memory
        const u32 sum = tmem + ((warp & 3) << 21);
        Turn acc;
        for (u32 r = 1; r <= emptied; ++r) {
            if (!wait_warp(&sh, &sh.acc_full[acc.s], acc.parity, g.wait_ns, g.flag)) break;
            tm_fence_after();
            const u32 from = sum + (1 + acc.s) * g.nt;
            for (u32 c = 0; c < g.nt; c += 16) {
                u32 v[16], t[16];
                tm_load8(from + c, v);
                tm_load8(from + c + 8, v + 8);
                tm_load8(sum + c, t);
                tm_load8(sum + c + 8, t + 8);
                tm_wait_load();
#pragma unroll
                for (u32 e = 0; e < 16; ++e) t[e] = __float_as_uint(__uint_as_float(t[e]) + __uint_as_float(v[e]));
                tm_store16(sum + c, t);
            }
            tm_wait_store();
            tm_fence_before();
            __syncwarp();
            if (elect_one()) mbar_arrive_own(&sh.acc_empty[acc.s]);
            __syncwarp();
            acc.next(g.accs - 1);
        }
    }
    if (parts > 1) cluster_wait();                 // every CTA of the cluster has started, its barriers are ready
    if (warp < WORK_WARPS) {
        // warps w and w + 4 read the same lanes of tensor memory, every other chunk of columns
        const u32 quarter = warp & 3, half = warp >> 2, row = quarter * 32 + (threadIdx.x & 31);
        const u32 lanes = tmem + ((quarter * 32) << 16);
        const u64 m = (u64)mt * PR_TILE + row;
        const float bias = g.turned ? column_bias(g.end, m) : 0.f;
        const bool ok = wait_warp(&sh, &sh.done, 0, g.wait_ns, g.flag);
        if (emptied) work_barrier();               // warps 4..7 have added up theirs
        tm_fence_after();
        u32 turn = 0;
        auto take = [&](auto width, u32 c, float (&f)[decltype(width)::value]) {
            constexpr u32 W = decltype(width)::value;
            auto load = [&](u32 at, u32* v, auto columns) {
                if constexpr (decltype(columns)::value == 32) {
                    tm_load32(at, v);
                } else {
#pragma unroll
                    for (u32 i = 0; i < decltype(columns)::value; i += 8) tm_load8(at + i, v + i);
                }
            };
            constexpr u32 STEP = W < 16 ? W : 16;                          // more does not fit the registers
            const std::integral_constant<u32, STEP> step;
            __syncwarp();
            if (RUNS && runs == 2) {               // both on the same way
                u32 v[W], t[STEP];
                load(lanes + c, v, width);
                load(lanes + g.nt + c, t, step);
                tm_wait_load();
#pragma unroll
                for (u32 e = 0; e < STEP; ++e) f[e] = __uint_as_float(v[e]) + __uint_as_float(t[e]);
                if constexpr (W > STEP) {
                    load(lanes + g.nt + c + STEP, t, step);
                    tm_wait_load();
#pragma unroll
                    for (u32 e = STEP; e < W; ++e) f[e] = __uint_as_float(v[e]) + __uint_as_float(t[e - STEP]);
                }
                return;
            }
            u32 v[W];
            if (runs) {
                load(lanes + c, v, width);
                tm_wait_load();
            }
#pragma unroll
            for (u32 e = 0; e < W; ++e) f[e] = runs ? __uint_as_float(v[e]) : 0.f;
            if constexpr (RUNS) {
                u32 slot = emptied % (ACCS - 1);                           // 0 where there are fewer accumulators
                for (u32 r = emptied + 1; r < runs; ++r) {
                    const u32 from = lanes + (1 + slot) * g.nt + c;
                    if (++slot == g.accs - 1) slot = 0;
#pragma unroll
                    for (u32 h = 0; h < W; h += STEP) {
                        u32 t[STEP];
                        __syncwarp();
                        load(from + h, t, step);
                        tm_wait_load();
#pragma unroll
                        for (u32 e = 0; e < STEP; ++e) f[h + e] += __uint_as_float(t[e]);
                    }
                }
            }
        };
        auto whole = [&](auto width) {            // 32 columns at a time where lanes have rows of y
            constexpr u32 W = decltype(width)::value;
            for (u32 c = half * W; c < cols; c += 2 * W) {
                float f[W];
                take(width, c, f);
                if constexpr (W == 32) end_rows<DT, OUT_BYTES>(g.end, &g.y, smem + warp * OUT_BYTES, turn, m, n0 + c, f);
                else end_column<DT, W>(g.end, n0 + c, m, min(W, cols - c), bias, f);
            }
        };
        auto send = [&](auto width) {              // the accumulator to shared memory
            constexpr u32 W = decltype(width)::value;
            for (u32 c = half * W; c < cols; c += 2 * W) {
                float f[W];
                take(width, c, f);
#pragma unroll
                for (u32 e = 0; e < W; ++e) if (c + e < g.nt) acc[(c + e) * PR_TILE + row] = f[e];
            }
        };
        auto join = [&](auto width) {              // own columns: their parts in ascending order
            constexpr u32 W = decltype(width)::value;
            for (u32 c = half * W; c < own_cols; c += 2 * W) {
                float f[W];
                for (u32 p = 0; p < parts; ++p) {
                    const float* from = p == part ? acc + (own + c) * PR_TILE + row : received + (p * g.per_owner + c) * PR_TILE + row;
#pragma unroll
                    for (u32 e = 0; e < W; ++e) {
                        const float v = c + e < own_cols ? from[e * PR_TILE] : 0.f;
                        f[e] = p ? f[e] + v : v;
                    }
                }
                if constexpr (W == 32) end_row<DT>(g.end, m, n0 + own + c, f);
                else end_column<DT, W>(g.end, n0 + own + c, m, min(W, own_cols - c), bias, f);
            }
        };
        if (parts == 1) {
            if (!g.turned) whole(std::integral_constant<u32, 32>());
            else if (g.nt > 16) whole(std::integral_constant<u32, 16>());
            else whole(std::integral_constant<u32, 8>());
        } else {
            send(std::integral_constant<u32, 8>());
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // the copies read what was just written
            work_barrier();
            if (warp == 0 && ok && elect_one()) {
                for (u32 i = 1; i < parts; ++i) {
                    const u32 to = part + i < parts ? part + i : part + i - parts, first = to * g.per_owner;
                    const u32 count = first < cols ? min(g.per_owner, cols - first) : 0;
                    if (count)
                        bulk_s2s(cluster_address(received + part * g.per_owner * PR_TILE, to), acc + first * PR_TILE, count * PR_TILE * 4,
                                 cluster_address(&sh.parts, to));
                }
            }
            __syncwarp();
            if (own_cols && !wait_warp(&sh, &sh.parts, 0, g.wait_ns, g.flag)) {
                if (elect_one()) {
                    for (u32 p = 0; p < parts; ++p) st_cluster_u32(cluster_address(const_cast<u32*>(&sh.late), p), 1);
                    asm volatile("fence.acq_rel.cluster;" ::: "memory");       // the arrival below is relaxed
                }
                __syncwarp();
            }
            if (!g.turned) join(std::integral_constant<u32, 32>());
            else join(std::integral_constant<u32, 8>());
        }
        end_rows_done();
        tm_fence_before();
    }
    __syncwarp();
    if (parts > 1) {                               // the others have what this CTA sent
        cluster_arrive();
        cluster_wait();
        // Unless one gave up: then all parts that will be sent are on their way by now, and the CTAs stay until they have landed.
        if (sh.late) {
            if (own_cols) drain_warp(&sh.parts, 0);
            cluster_arrive();
            cluster_wait();
        }
    }
    __syncthreads();
    tm_fence_after();
    if (warp == PRODUCT_WARP) tm_dealloc(tmem, g.tmem_cols);
}

template <int DT, bool RUNS>
bool launch_as(cudaStream_t s, const NarrowArgs& g, u32 blocks, u32 parts, u32 smem) {
    static std::atomic<u64> allowed{0};
    if (!allow_smem(product_kernel<DT, RUNS>, allowed, SMEM_MAX)) return false;
    return launch_chained(product_kernel<DT, RUNS>, blocks, THREADS, smem, parts, s, g);
}

// How a product is cut: which operand is on which side, rows of n per CTA, CTAs that share the columns of a tile.
struct Cut {
    bool turned;
    u32 nt, parts, boxes, stages, accs, tmem_cols, smem, ring_bytes, per_owner;
    float us;
    bool guess;                                    // the driver did not say how many clusters run at once
};

// Blocks that run at once in clusters of `parts`, one to an SM; 0 where the driver did not say.  Clusters stay within a group of SMs, whose sizes only
// the driver knows (which counts one block to an SM of a kernel that uses tensor memory, however little).
u32 at_once(int device, int sms, u32 parts) {
    if (parts == 1) return (u32)sms;
    static PerDevice<MAX_SPLIT + 1> known;
    return known.get(device, parts, [&]() -> u32 {
        static std::atomic<u64> allowed{0};
        if (!allow_smem(product_kernel<DT_F32, true>, allowed, SMEM_MAX)) return 0;
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = parts;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.gridDim = dim3((u32)sms / parts * parts);
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = SMEM_MAX;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, product_kernel<DT_F32, true>, &cfg) != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        return clusters > 0 ? (u32)clusters * parts : 1;       // 1: nothing is split so
    });
}

// Stages of a run; accumulators for so many stages.
u32 run_of(u32 boxes) { return PR_RUN / (PR_K * boxes); }
u32 accs_of(u32 steps, u32 boxes) { return steps <= run_of(boxes) ? 1 : steps <= 2 * run_of(boxes) ? 2 : ACCS; }

// About how long a cut takes, in us, as measured: 3.2 for a launch, its first copies and the end; what an SM fetches, 135 bytes a ns (a CTA
// alone 75 of the larger operand where it comes from memory, which gives 6500 in all, or 5600 to fewer than three CTAs on two SMs; L2 15000), and at least the
// products (1.05 ns for a row of n and 64 columns); 10 ns for a column of the accumulator that lanes write across rows of y and 4 along
// them; 1 and 0.25 a part and 6 ns a column for the exchange within a cluster; 6 for a further turn of the SMs.
Cut find_cut(const ProductCall& c, bool y_vec) {
    Cut best{};
    best.us = 1e30f;
    bool guess = false;
    const u32 k_boxes = (u32)((c.a.k + PR_K - 1) / PR_K);
    const float memory = (float)(c.a.rows + c.b.rows) * (float)c.a.k * 2.f, alone = memory > 60e6f ? 75e3f : 135e3f, all = memory > 60e6f ? 6.5e6f : 15e6f;
    for (int side = 0; side < 2; ++side) {
        const bool turned = side == 0;
        if (!turned && !y_vec) break;              // rows of y that start anywhere are written across
        const ProductOperand& m = turned ? c.b : c.a;
        const ProductOperand& n = turned ? c.a : c.b;
        const u64 m_tiles = (m.rows + PR_TILE - 1) / PR_TILE;
        for (u32 want : {16u, 32u, 48u, 64u, 96u, 128u}) {
            if (!turned && want % 32) continue;    // whole blocks of 32 columns
            if (want > 16 && want >= n.rows + 32) break;
            const u64 tiles = m_tiles * ((n.rows + want - 1) / want);
            const u32 n_bytes = n.along_k ? want * PR_K * 2 : (want + PR_CHUNK - 1) / PR_CHUNK * PR_CHUNK_BYTES;
            for (u32 parts = 1; parts <= MAX_SPLIT && (parts == 1 || (k_boxes >= parts && tiles * parts <= (u64)c.sms * 2)); ++parts) {
                Cut cut{turned, want, parts, BOXES_MAX, 0, 1, 0, 0, 0, 0, 0.f, false};
                cut.per_owner = (want + parts - 1) / parts;
                if (!turned) cut.per_owner = (cut.per_owner + 31) & ~31u;
                const u32 sums = parts > 1 ? parts * cut.per_owner * PR_TILE * 4 : 0, own = parts > 1 ? want * PR_TILE * 4 : turned ? 0 : WORK_WARPS * OUT_BYTES;
                const u32 box = M_BYTES + n_bytes;
                auto room_for = [&](u32 room, u32 boxes) { return room > sums + 1024 ? (room - sums - 1024) / (box * boxes) : 0u; };
                auto steps_of = [&](u32 boxes) { return (k_boxes + boxes - 1) / boxes / parts + ((k_boxes + boxes - 1) / boxes % parts != 0); };
                // Two CTAs to an SM where there are more than one each; two boxes of 64 columns to a stage (waiting for one and handing it back
                // cost 250 cycles, whatever it holds), or one: the first of these that leaves enough stages.
                bool two = false;
                u32 stages = 0;
                for (u32 way = tiles * parts > (u64)c.sms && want * accs_of(steps_of(BOXES_MAX), BOXES_MAX) <= 128 ? 0 : 2; way < 4; ++way) {
                    two = way < 2;
                    cut.boxes = way % 2 ? 1 : BOXES_MAX;
                    stages = room_for(two ? SMEM_MAX / 2 - 1024 : SMEM_MAX, cut.boxes);
                    if (stages >= (cut.boxes == 1 ? 4 : 3) || stages >= steps_of(cut.boxes)) break;
                }
                if (!stages) continue;
                if (stages > STAGES_MAX) stages = STAGES_MAX;
                const u32 steps = steps_of(cut.boxes);
                if (parts > 1 && (k_boxes + cut.boxes - 1) / cut.boxes < parts) continue;
                cut.stages = stages < steps ? stages : steps ? steps : 1;
                cut.ring_bytes = cut.stages * cut.boxes * box > own ? cut.stages * cut.boxes * box : own;
                cut.smem = cut.ring_bytes + sums + 1024;
                if (cut.smem > SMEM_MAX) continue;
                cut.accs = accs_of(steps, cut.boxes);
                cut.tmem_cols = 32;
                while (cut.tmem_cols < want * cut.accs) cut.tmem_cols *= 2;
                const u32 least = cut.tmem_cols >= 512 ? SMEM_MAX : cut.tmem_cols * (SMEM_SM / 512);
                if (cut.smem < least) cut.smem = least;
                if (cut.smem < SMEM_LEAST) cut.smem = SMEM_LEAST;
                if (cut.smem > SMEM_MAX / 2 - 1024) two = false;
                const u64 room = (u64)at_once(c.device, c.sms, parts) * (two ? 2 : 1), blocks = tiles * parts;
                guess |= room == 0;
                if (parts > 1 && blocks > room) continue;
                const u64 per_sm = (blocks + c.sms - 1) / c.sms, turns = (blocks + room - 1) / room;
                const float beside = two && per_sm > 1 ? 2.f : 1.f, rate = fminf(alone, 135e3f / beside);
                const float near = 135e3f / beside, fetch = m.rows >= n.rows ? M_BYTES / rate + n_bytes / near : M_BYTES / near + n_bytes / rate;
                const float step = cut.boxes * fmaxf(fetch, beside * want * 1.05e-3f);
                const float whole = memory > 60e6f && blocks * 2 < (u64)c.sms * 3 ? 1.16f * memory / all : memory / all;
                cut.us = 3.2f + fmaxf((float)turns * steps * step, whole) + (turns - 1) * 6.f +
                         (float)turns * want / parts * (turned ? 0.010f : 0.004f) + (parts > 1 ? 1.f + 0.25f * parts + 0.006f * want : 0.f);
                if (cut.us < best.us) best = cut;
            }
        }
    }
    best.guess = guess;
    return best;
}

// The search takes 10 us of host time: the cuts of the last shapes are kept (a function of the device and the sizes alone).
Cut best_cut(const ProductCall& c, bool y_vec) {
    struct Entry {
        u64 a_rows = 0, b_rows = 0, k = 0;
        u32 how = 0;
        int device = 0;
        Cut cut;
    };
    thread_local Entry kept[32];
    const u32 how = 1u | (c.a.along_k ? 2u : 0u) | (c.b.along_k ? 4u : 0u) | (y_vec ? 8u : 0u) | (u32)c.sms << 4;
    Entry& e = kept[((c.a.rows * 31 + c.b.rows) * 31 + c.a.k * 7 + how) * 0x9e3779b97f4a7c15ull >> 59];
    if (e.how == how && e.device == c.device && e.a_rows == c.a.rows && e.b_rows == c.b.rows && e.k == c.a.k) return e.cut;
    const Cut cut = find_cut(c, y_vec);
    if (!cut.guess) e = Entry{c.a.rows, c.b.rows, c.a.k, how, c.device, cut};
    return cut;
}

bool launch_narrow(cudaStream_t s, const ProductCall& c, const EndArgs& end, const Cut& cut) {
    NarrowArgs g;
    g.end = end;
    g.turned = cut.turned;
    const ProductOperand& m = g.turned ? c.b : c.a;
    const ProductOperand& n = g.turned ? c.a : c.b;
    g.nt = cut.nt;
    g.n_tiles = (u32)((n.rows + g.nt - 1) / g.nt);
    g.k_boxes = (u32)((m.k + PR_K - 1) / PR_K);
    const u64 m_tiles = (m.rows + PR_TILE - 1) / PR_TILE;
    g.n_bytes = n.along_k ? g.nt * PR_K * 2 : (g.nt + PR_CHUNK - 1) / PR_CHUNK * PR_CHUNK_BYTES;
    g.boxes = cut.boxes;
    g.per_owner = cut.per_owner;
    g.stages = cut.stages;
    g.ring_bytes = cut.ring_bytes;
    g.accs = cut.accs;
    const u32 k_steps = (g.k_boxes + cut.boxes - 1) / cut.boxes, steps = k_steps / cut.parts + (k_steps % cut.parts != 0);
    g.runs = (steps + run_of(cut.boxes) - 1) / run_of(cut.boxes);
    g.run = g.runs ? (steps + g.runs - 1) / g.runs : 0;
    g.runs = g.run ? (steps + g.run - 1) / g.run : 0;
    g.tmem_cols = cut.tmem_cols;
    if (g.k_boxes && (!product_map(&g.m, m, PR_TILE, c.dtype) || !product_map(&g.n, n, g.nt, c.dtype))) return false;
    if (!g.turned && cut.parts == 1 && !result_map(&g.y, c.end.y)) return false;
    g.m_along_k = m.along_k;
    g.n_along_k = n.along_k;
    g.bf16 = c.dtype == DT_BF16;
    g.wait_ns = c.wait_ns;
    g.flag = c.flag;
    const u32 blocks = (u32)(m_tiles * g.n_tiles) * cut.parts;
    auto launch = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if constexpr (DT != DT_F32) if (cut.accs == 1) return launch_as<DT, false>(s, g, blocks, cut.parts, cut.smem);
        return launch_as<DT, true>(s, g, blocks, cut.parts, cut.smem);
    };
    return c.end.y.dtype == DT_F32 ? launch(std::integral_constant<int, DT_F32>()) : c.end.y.dtype == DT_F16 ? launch(std::integral_constant<int, DT_F16>())
                                                                                                           : launch(std::integral_constant<int, DT_BF16>());
}

// Eight values of a row at a time: 16 bytes of the result, cut out of the two aligned words that hold them.
constexpr u32 TIDY_THREADS = 256;
__global__ void __launch_bounds__(TIDY_THREADS) tidy_kernel(const unsigned short* __restrict__ x, u64 rows, u64 cols, u64 stride, unsigned short* __restrict__ to, u64 pitch) {
    wait_for_previous();
    let_next_start();
    const u64 words = pitch / 8, total = rows * words;
    for (u64 i = (u64)blockIdx.x * TIDY_THREADS + threadIdx.x; i < total; i += (u64)gridDim.x * TIDY_THREADS) {
        const u64 row = i / words, c = (i - row * words) * 8;
        const unsigned short* r = x + row * stride;
        const char* p = reinterpret_cast<const char*>(r + c);
        const u32 shift = (u32)(reinterpret_cast<uintptr_t>(p) & 15);
        p -= shift;
        uint4 q;
        // every byte that is read belongs to the row
        if (p >= reinterpret_cast<const char*>(r) && p + 32 <= reinterpret_cast<const char*>(r + cols)) {
            q = cut16(__ldg(reinterpret_cast<const uint4*>(p)), __ldg(reinterpret_cast<const uint4*>(p) + 1), shift);
        } else {
            unsigned short* h = reinterpret_cast<unsigned short*>(&q);
#pragma unroll
            for (u32 e = 0; e < 8; ++e) h[e] = c + e < cols ? r[c + e] : 0;
        }
        *reinterpret_cast<uint4*>(to + row * pitch + c) = q;
    }
}

}  // namespace

u64 tidy_pitch(u64 cols) { return (cols + 63) & ~63ull; }

void launch_tidy(int sms, cudaStream_t s, const Matrix& m, void* to) {
    const u64 pitch = tidy_pitch(m.cols), blocks = (m.rows * (pitch / 8) + TIDY_THREADS - 1) / TIDY_THREADS, most = (u64)sms * 32;
    launch_chained(tidy_kernel, (u32)(blocks < most ? blocks : most), TIDY_THREADS, 0, 0, s, static_cast<const unsigned short*>(m.p), m.rows, m.cols, m.stride,
                   static_cast<unsigned short*>(to), pitch);
}

namespace {
bool encode_map(CUtensorMap* map, CUtensorMapDataType type, const void* p, u64 inner, u64 outer, u64 pitch, u32 box_inner, u32 box_outer, CUtensorMapSwizzle swizzle) {
    static const auto encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(f);
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {inner, outer}, strides[1] = {pitch};
    const cuuint32_t box[2] = {box_inner, box_outer}, one[2] = {1, 1};
    return encode(map, type, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
CUtensorMapDataType map_type(int dtype) {
    return dtype == DT_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}
}  // namespace

bool product_map(CUtensorMap* map, const ProductOperand& o, u32 box_rows, int dtype) {
    return encode_map(map, map_type(dtype), o.p, o.along_k ? o.k : o.rows, o.along_k ? o.rows : o.k, o.stride * 2, PR_K, o.along_k ? box_rows : PR_K, CU_TENSOR_MAP_SWIZZLE_128B);
}

bool result_map(CUtensorMap* map, const Matrix& y) {
    const u64 size = y.dtype == DT_F32 ? 4 : 2, pitch = y.rows == 1 ? (y.cols * size + 15) & ~15ull : y.stride * size;
    return encode_map(map, map_type(y.dtype), y.p, y.cols, y.rows, pitch, 32, 32, size == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

EndArgs end_args(const ProductEnd& e) {
    EndArgs g;
    auto size = [](int dtype) { return dtype == DT_F32 ? 4ull : 2ull; };
    auto on = [&](const Matrix& m, u64 bytes) { return ((reinterpret_cast<uintptr_t>(m.p) | (m.rows == 1 ? 0 : m.stride * size(m.dtype))) & (bytes - 1)) == 0; };
    g.y = e.y.p;
    g.stride = e.y.stride;
    g.rows = e.y.rows;
    g.cols = e.y.cols;
    g.bias = e.bias.p;
    g.bias_dtype = e.bias.dtype;
    g.act = e.act;
    g.residual = e.residual.p;
    g.residual_stride = e.residual.stride;
    g.residual_dtype = e.residual.dtype;
    g.kept = e.kept.p;
    g.kept_stride = e.kept.stride;
    g.kept_dtype = e.kept.dtype;
    if (e.kept.p && e.kept.dtype == DT_ACT8) g.k8 = Kept(e.kept.p, e.y.rows, e.y.cols);
    auto level = [&](const Matrix& m) { return on(m, 32) ? 2u : on(m, 16) ? 1u : 0u; };
    g.y_vec = level(e.y);
    g.bias_vec = e.bias.p && (reinterpret_cast<uintptr_t>(e.bias.p) & 15) == 0;
    g.residual_vec = e.residual.p && on(e.residual, 16);
    g.kept_vec = !e.kept.p ? 0 : e.kept.dtype == DT_ACT8 ? ((reinterpret_cast<uintptr_t>(e.kept.p) & 31) == 0 ? 2 : 1) : level(e.kept);
    return g;
}

bool launch_product(cudaStream_t s, const ProductCall& c) {
    const EndArgs end = end_args(c.end);
    const Cut cut = best_cut(c, end.y_vec != 0);
    // tiles of 256 x 256 where both sides have more than one of 128
    if (c.a.k && c.a.rows > PR_TILE && c.b.rows > PR_TILE && product_wide_us(c) < cut.us) return launch_product_wide(s, c);
    return launch_narrow(s, c, end, cut);
}

}  // namespace excp
