// Product of two microscaled 4-bit matrices: y[a row, b row] = scales * sum over columns (+ bias), fp32 sums.
// This file: few rows on one side (the tokens of a decoding step); mx4_matmul_wide.cu: many rows on both.
//
// Bound: the bytes of the larger matrix; for small ones the chain launch, copy, product, exchange.  (4096 -> 11008, blocks of 16,
// 25 MB: one token quantised here 7.6 us, 16 packed tokens 8.4 us, 128 tokens 10.9 us; 2048 -> 50304, 55 MB, 16 tokens 12.5 us,
// 4.4 TB/s; 128 columns alone 3.3 us.)  Its rows go on the M side of the tensor core (128 per tile), the few rows on the N
// side, which takes them in steps of 8.  Several CTAs share an SM, and the columns of a tile are split over a cluster so
// that every SM streams; each CTA sends its part of a column of the result to the CTA that owns the column (distributed shared
// memory), which adds them in a fixed order.
//
// Roles: warp 4 fetches (contiguous bulk copies: the packed layout is the tensor core's), warp 5 issues the matrix
// instructions; warps 0..3 bring the block scales to tensor memory and write the result.  Where the few rows come as plain
// values (linear), warps 0..3 first quantise them into shared memory, each CTA the columns it needs, while the first tiles
// are on their way: a launch less.
// Every wait for a copy, a product or another warp is bounded; where one runs out the CTA raises the handle's flag, lets its copies land and
// leaves.  The two that hardware gives no limit, for tensor memory and at the cluster's barrier, depend only on CTAs whose own
// waits are bounded.
#include <type_traits>

#include "mx4_codes.cuh"
#include "mx4_pipe.cuh"

namespace excp {
namespace {

constexpr int WORK_WARPS = 4;                      // scales, quantisation, result
constexpr u32 FETCH_WARP = WORK_WARPS, PRODUCT_WARP = WORK_WARPS + 1;
constexpr int THREADS = (WORK_WARPS + 2) * 32;
constexpr int STAGES = 3;
constexpr u32 CODES = MX4_ROWS * 128;
constexpr u32 MAX_SPLIT = 8;
constexpr u32 RAW_TASKS = 24;                      // plain rows x column tiles that a CTA quantises itself
constexpr u32 RAW_ROWS = 16;                       // and at most so many (at most 32: one column of tensor memory holds their scales)
constexpr u32 SMEM_MAX = 227 * 1024 - 1024;        // dynamic shared memory of a block, beside what the kernel has of its own
// Shared memory that the rows a CTA quantises take at most: rounding up to 8 makes them 8 times as many where there is one.
constexpr u32 RAW_BYTES = 8 * RAW_TASKS * (128 + mx4_pieces(MX4_E4M3_16) * 4);
static_assert(STAGES * (CODES + mx4_scale_bytes(MX4_E4M3_16)) + 1024 + (RAW_ROWS + MAX_SPLIT) * MX4_ROWS * 4 + 1024 + RAW_BYTES <= SMEM_MAX, "shared memory of the fused product");

struct NarrowArgs {
    Mx4Operand m;                                  // M side
    Mx4Operand n;                                  // N side, packed (not RAW)
    const void* x;                                 // N side as plain values (RAW)
    u64 x_stride, cols;
    u32 x_vec;                                     // its rows start on 16 bytes
    u32 col_tiles, nt, n_tiles;                    // rows of n per CTA: a multiple of 8, at most 128
    u32 x_codes, x_scales;                         // where the quantised rows lie in shared memory (RAW)
    void* y;
    u64 stride;                                    // y[row of n, row of m]
    const float* bias;                             // per row of m
    u32 sums;                                      // where the parts of the CTA's columns lie in shared memory
    u32 stage_bytes, tmem_cols;
    u32 early;                                     // the launch before packs n, and m may be fetched before it ends
    u64 wait_ns;
    u32* flag;
};

struct Shared {
    unsigned long long full[STAGES];               // copies have landed
    unsigned long long ready[STAGES];              // and the scales are in tensor memory (and plain rows quantised)
    unsigned long long empty[STAGES];              // the stage has been multiplied
    unsigned long long done;
    u32 tmem;
    volatile u32 abort;
};

__device__ __forceinline__ void work_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// Columns 8 lane .. 8 lane + 7 of column tile `ct` of a plain row, 0 past the end.
template <typename T>
__device__ __forceinline__ void load_part(const NarrowArgs& g, u64 row, u32 ct, u32 lane, float v[8]) {
    const u64 c0 = (u64)ct * MX4_COLS + lane * 8;
    const T* p = static_cast<const T*>(g.x) + row * g.x_stride + c0;
    if (row < g.n.rows && g.x_vec && c0 + 8 <= g.cols) {
        load8(p, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = row < g.n.rows && c0 + k < g.cols ? wget(p, k) : 0.f;
    }
}

// One plain row of a column tile -> its codes, and its scales as one word per piece, `rows` words apart.
template <int FMT>
__device__ __forceinline__ void quantize_row(float (&v)[8], u32 r, u32 lane, float gx, unsigned char* codes, u32* scales, u32 rows) {
    u32 top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    if (FMT == MX4_E8M0_32) top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const u32 byte = FMT == MX4_E8M0_32 ? scale_e8m0(v, top) : scale_e4m3(v, top, gx, 6.f * gx);
    *reinterpret_cast<u32*>(codes + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + ((lane & 3) << 2)) = codes_of<FMT>(v);
    constexpr u32 PER = mx4_block(FMT) / 8, PIECES = mx4_pieces(FMT);
    const u32 piece = min(lane, PIECES - 1);
    const u32 word = scale_word<FMT>(byte, piece * 4 * PER);
    if (lane < PIECES) scales[piece * rows + r] = word;
}

template <int FMT, int DT, int XT>                 // XT: type of the plain rows, -1 = both sides packed
__global__ void __launch_bounds__(THREADS, 3) narrow_kernel(const __grid_constant__ NarrowArgs g) {
    constexpr bool RAW = XT >= 0;
    constexpr u32 PIECES = mx4_pieces(FMT), SB = mx4_scale_bytes(FMT), SF_COLS = PIECES * 8;
    typedef typename ElemOf<RAW ? XT : DT_F32>::type X;
    typedef typename ElemOf<DT>::type T;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared sh;
    const u32 part = cluster_rank(), parts = cluster_size();
    // the swizzle goes by address: stages start on 1024 bytes (the same offset in every CTA)
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const u32 warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const u32 tile = blockIdx.x / parts, mt = tile / g.n_tiles, ntile = tile - mt * g.n_tiles;
    const u32 k0 = (u32)((u64)g.col_tiles * part / parts), k1 = (u32)((u64)g.col_tiles * (part + 1) / parts);
    const u32 per_owner = (g.nt + parts - 1) / parts;          // columns of the result per CTA of the cluster
    // a stage: tile of m (codes, scales), packed rows of n (codes), their scales
    const u32 n_codes = CODES + SB, n_scales = n_codes + g.nt * 128;

    if (!g.early) wait_for_previous();
    let_next_start();
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.ready[s], WORK_WARPS); mbar_init(&sh.empty[s], 1); }
        mbar_init(&sh.done, 1);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == PRODUCT_WARP) tm_alloc(&sh.tmem, g.tmem_cols);
    tm_fence_before();
    __syncthreads();
    if (parts > 1) cluster_arrive();
    tm_fence_after();
    const u32 tmem = sh.tmem;
    bool ok = true;                                // this warp's waits were all met

    if (warp == FETCH_WARP) {
        const u32 hm = mx4_tile_height(g.m.rows, mt), hn = RAW ? 0 : mx4_tile_height(g.n.rows, ntile);
        const unsigned char* pm = g.m.p + mx4_tile_offset(g.m.rows, g.col_tiles, FMT, mt, k0);
        const unsigned char* pn = RAW ? nullptr : g.n.p + mx4_tile_offset(g.n.rows, g.col_tiles, FMT, ntile, k0);
        const u32 bytes = hm * 128 + SB + (RAW ? 0 : hn * 128 + SB);
        Ring<STAGES> ring;
        u32 filled = 0;
        auto fetch_m = [&](u32 s) {                // announces the whole stage
            unsigned char* st = smem + s * g.stage_bytes;
            if (elect_one()) {
                mbar_arrive_expect_tx(&sh.full[s], bytes);
                if (hm == MX4_ROWS) {
                    bulk_g2s(st, pm, CODES + SB, &sh.full[s]);
                } else {
                    bulk_g2s(st, pm, hm * 128, &sh.full[s]);
                    bulk_g2s(st + CODES, pm + hm * 128, SB, &sh.full[s]);
                }
            }
            __syncwarp();
            pm += hm * 128 + SB;
        };
        auto fetch_n = [&](u32 s) {
            unsigned char* st = smem + s * g.stage_bytes;
            if (elect_one()) {
                bulk_g2s(st + n_codes, pn, hn * 128, &sh.full[s]);
                bulk_g2s(st + n_scales, pn + hn * 128, SB, &sh.full[s]);
            }
            __syncwarp();
            pn += hn * 128 + SB;
        };
        // the first stages' tiles of m, before the launch that may just be packing n has ended
        const u32 first = min((u32)STAGES, k1 - k0);
        for (u32 s = 0; s < first; ++s) fetch_m(s);
        if (!RAW) {
            if (g.early) wait_for_previous();
            for (u32 s = 0; s < first; ++s) fetch_n(s);
        }
        for (u32 s = 0; s < first; ++s, ++filled) ring.next();
        for (u32 k = k0 + first; k < k1; ++k) {
            if (!(ok = wait_warp(&sh, &sh.empty[ring.s], ring.parity ^ 1, g.wait_ns, g.flag))) break;
            fetch_m(ring.s);
            if (!RAW) fetch_n(ring.s);
            ++filled;
            ring.next();
        }
        // no copy may be in flight when the CTA leaves: the last turn of every stage that was filled
        for (u32 i = 0; i < STAGES && i < filled; ++i) {
            if (ring.s == 0) { ring.s = STAGES; ring.parity ^= 1; }
            --ring.s;
            drain_warp(&sh.full[ring.s], ring.parity);
        }
    } else if (warp == PRODUCT_WARP) {
        const u32 idesc = (1u << 7) | (1u << 10) | ((g.nt >> 3) << 17) | (FMT == MX4_E8M0_32 ? 1u << 23 : 0u) | (8u << 24);
        Ring<STAGES> ring;
        for (u32 k = k0; k < k1; ++k) {
            if (!(ok = wait_warp(&sh, &sh.ready[ring.s], ring.parity, g.wait_ns, g.flag))) break;
            tm_fence_after();
            const u32 st = smem_u32(smem) + ring.s * g.stage_bytes;
            const u32 sa = tmem + g.nt + ring.s * SF_COLS, sb = sa + PIECES * 4;
            const u64 da = desc_swizzled(st), db = desc_swizzled(RAW ? smem_u32(smem) + g.x_codes + (k - k0) * g.nt * 128 : st + n_codes);
            if (elect_one()) {
#pragma unroll
                for (u32 i = 0; i < 4; ++i) {      // 64 columns = 32 bytes of codes each
                    if (FMT == MX4_E4M3_16) {
                        tm_mma_block16(tmem, da + 2 * i, db + 2 * i, idesc, sa + i * 4, sb + i * 4, k > k0 || i);
                    } else {
                        const u32 half = (i & 1) * 2, j = i >> 1;          // a piece serves two instructions: its bytes 0, 1, then 2, 3
                        tm_mma_block32(tmem, da + 2 * i, db + 2 * i, idesc | (half << 4) | (half << 29), sa + j * 4, sb + j * 4, k > k0 || i);
                    }
                }
                tm_commit(&sh.empty[ring.s]);
            }
            __syncwarp();
            ring.next();
        }
        if (elect_one()) tm_commit(&sh.done);
        __syncwarp();
        drain_warp(&sh.done, 0);                   // what has been issued is done before tensor memory goes
    } else {
        if (RAW) {
            // Row r of column tile k0 + t is task t * rows + r; the rows past the end stay as they are (only their own
            // results, which are not written, would see them).
            const float gx = g.n.scale ? __ldg(g.n.scale) : 1.f;
            const u32 rows = (u32)g.n.rows, tasks = (k1 - k0) * rows;
            constexpr u32 AHEAD = 2;
            float v[AHEAD][8];
            auto fetch = [&](u32 i, float (&to)[8]) {
                if (i < tasks) load_part<X>(g, i % rows, k0 + i / rows, lane, to);
            };
#pragma unroll
            for (u32 a = 0; a < AHEAD; ++a) fetch(warp + a * WORK_WARPS, v[a]);
            for (u32 i = warp; i < tasks; i += AHEAD * WORK_WARPS) {
#pragma unroll
                for (u32 a = 0; a < AHEAD; ++a) {
                    const u32 at = i + a * WORK_WARPS;
                    if (at >= tasks) break;
                    const u32 t = at / rows, r = at - t * rows;
                    quantize_row<FMT>(v[a], r, lane, gx, smem + g.x_codes + t * g.nt * 128,
                                      reinterpret_cast<u32*>(smem + g.x_scales) + t * PIECES * g.nt, g.nt);
                    fetch(at + AHEAD * WORK_WARPS, v[a]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");         // the tensor core reads what was just written
            work_barrier();
        }
        Ring<STAGES> ring;
        for (u32 k = k0; k < k1; ++k) {
            if (!(ok = wait_warp(&sh, &sh.full[ring.s], ring.parity, g.wait_ns, g.flag))) break;
            const unsigned char* st = smem + ring.s * g.stage_bytes;
            const uint4* from = reinterpret_cast<const uint4*>(st + CODES) + lane;
            // each stage has scale columns of its own, free again when the stage is
            const u32 sa = tmem + ((warp * 32) << 16) + g.nt + ring.s * SF_COLS;
            uint4 a[2 * PIECES];
#pragma unroll
            for (u32 j = 0; j < PIECES; ++j) a[j] = from[j * 32];
            if (RAW) {                             // at most 32 rows: the first of the four columns
                const u32* words = reinterpret_cast<const u32*>(smem + g.x_scales) + (k - k0) * PIECES * g.nt;
#pragma unroll
                for (u32 j = 0; j < PIECES; ++j) a[PIECES + j] = make_uint4(lane < g.nt ? words[j * g.nt + lane] : 0u, 0u, 0u, 0u);
            } else {
                const uint4* from_n = reinterpret_cast<const uint4*>(st + n_scales) + lane;
#pragma unroll
                for (u32 j = 0; j < PIECES; ++j) a[PIECES + j] = from_n[j * 32];
            }
            if (FMT == MX4_E4M3_16) tm_store32(sa, reinterpret_cast<const u32*>(a));
            else tm_store16(sa, reinterpret_cast<const u32*>(a));
            tm_wait_store();
            tm_fence_before();
            __syncwarp();
            if (elect_one()) mbar_arrive_own(&sh.ready[ring.s]);
            ring.next();
        }
        if (ok) ok = wait_warp(&sh, &sh.done, 0, g.wait_ns, g.flag);
        tm_fence_after();
    }

    const TensorScales by = tensor_scales(g.m.scale, g.n.scale);
    const u64 n0 = (u64)ntile * MX4_ROWS;
    const u32 cols = (u32)min((u64)g.nt, g.n.rows - n0);       // of the result
    // thread t of the work warps has row t of m's tile
    const u32 t = threadIdx.x;
    const u64 m = (u64)mt * MX4_ROWS + t;
    T* const y = static_cast<T*>(g.y) + n0 * g.stride + m;
    const float bias = g.bias && warp < WORK_WARPS && m < g.m.rows ? __ldg(g.bias + m) : 0.f;
    // A warp per scheduler: no branches between the columns, so that they overlap.
    auto put = [&](auto width, const float (&sum)[decltype(width)::value], u32 c, u32 step) {    // columns c, c + step, ...
        constexpr u32 W = decltype(width)::value;
        if (m >= g.m.rows) return;
        float r[W];
#pragma unroll
        for (u32 i = 0; i < W; ++i) r[i] = sum[i] * by.first;
        if (by.second != 1.f) {
#pragma unroll
            for (u32 i = 0; i < W; ++i) r[i] *= by.second;
        }
        if (g.bias) {
#pragma unroll
            for (u32 i = 0; i < W; ++i) r[i] += bias;
        }
        T* const p = y + c * g.stride;
        const u64 jump = step * g.stride;
        if (c + (W - 1) * step < cols) {
#pragma unroll
            for (u32 i = 0; i < W; ++i) wput(p + i * jump, 0, r[i]);
        } else {
#pragma unroll
            for (u32 i = 0; i < W; ++i) if (c + i * step < cols) wput(p + i * jump, 0, r[i]);
        }
    };
    auto take = [&](auto width, u32 c) {           // that many columns of the accumulator
        constexpr u32 W = decltype(width)::value;
        u32 v[W];
#pragma unroll
        for (u32 i = 0; i < W; i += 32) {
            if constexpr (W >= 32) tm_load32(tmem + ((warp * 32) << 16) + c + i, v + i);
            else tm_load8(tmem + ((warp * 32) << 16) + c + i, v + i);
        }
        tm_wait_load();
        float f[W];
#pragma unroll
        for (u32 i = 0; i < W; ++i) f[i] = k0 < k1 ? __uint_as_float(v[i]) : 0.f;
        if (parts == 1) {
            put(width, f, c, 1);
        } else {
            // column c belongs to CTA c % parts, which has a place for this CTA's part of it
            u32 owner = c % parts, at = ((part * per_owner + c / parts) * MX4_ROWS + t) * 4;
#pragma unroll
            for (u32 i = 0; i < W; ++i) {
                if (c + i < cols) st_cluster(cluster_address(smem + g.sums, owner) + at, f[i]);
                if (++owner == parts) { owner = 0; at += MX4_ROWS * 4; }
            }
        }
    };
    if (parts > 1) cluster_wait();                 // every CTA of the cluster has started
    if (warp < WORK_WARPS) {
        u32 c = 0;
        for (; c + 64 <= g.nt; c += 64) take(std::integral_constant<u32, 64>(), c);
        for (; c < g.nt; c += 8) take(std::integral_constant<u32, 8>(), c);
        tm_fence_before();
    }
    __syncwarp();
    if (parts > 1) {
        cluster_arrive_release();
        cluster_wait();
        if (warp < WORK_WARPS) {
            const float* own = reinterpret_cast<const float*>(smem + g.sums) + t;
            auto join = [&](auto width, u32 j) {   // own columns j ..: their parts in ascending order
                constexpr u32 W = decltype(width)::value;
                float f[W];
#pragma unroll
                for (u32 i = 0; i < W; ++i) f[i] = own[min(j + i, per_owner - 1) * MX4_ROWS];
                for (u32 p = 1; p < parts; ++p) {
#pragma unroll
                    for (u32 i = 0; i < W; ++i) f[i] += own[(p * per_owner + min(j + i, per_owner - 1)) * MX4_ROWS];
                }
                put(width, f, part + j * parts, parts);
            };
            u32 j = 0;
            for (; j + 8 <= per_owner; j += 8) join(std::integral_constant<u32, 8>(), j);
            for (; j < per_owner; j += 2) join(std::integral_constant<u32, 2>(), j);
        }
    }
    __syncwarp();
    __syncthreads();
    tm_fence_after();
    if (warp == PRODUCT_WARP) tm_dealloc(tmem, g.tmem_cols);
}

template <int FMT, int DT, int XT>
bool launch_as(cudaStream_t s, const NarrowArgs& g, u32 parts, u32 smem) {
    static std::atomic<u64> allowed{0};
    if (!allow_smem(narrow_kernel<FMT, DT, XT>, allowed, SMEM_MAX)) return false;
    return launch_chained(narrow_kernel<FMT, DT, XT>, mx4_row_tiles(g.m.rows) * g.n_tiles * parts, THREADS, smem, parts, s, g);
}

template <int XT>
bool launch_typed(cudaStream_t s, const NarrowArgs& g, u32 parts, u32 smem, int fmt, int dtype) {
#define EXCP_MM(DT) (fmt == MX4_E4M3_16 ? launch_as<MX4_E4M3_16, DT, XT>(s, g, parts, smem) : launch_as<MX4_E8M0_32, DT, XT>(s, g, parts, smem))
    return dtype == DT_F32 ? EXCP_MM(DT_F32) : dtype == DT_F16 ? EXCP_MM(DT_F16) : EXCP_MM(DT_BF16);
#undef EXCP_MM
}

u32 split(int sms, u64 m_tiles, u64 n_tiles, u32 nt, u32 col_tiles) {
    // Two CTAs per SM as long as there are columns to split, if that pays: a column tile takes a CTA about 0.3 us, exchanging the
    // parts 1.5 us and 0.06 us per row.  (4096 -> 11008: 8 rows whole 8.3 us, in three parts 7.6; 64 rows whole 9.2, in two
    // parts 18.7.)
    u32 best = 1;
    float least = 0.3f * col_tiles;
    for (u32 parts = 2; parts <= MAX_SPLIT && parts <= col_tiles && m_tiles * n_tiles * parts <= (u64)sms * 2; ++parts) {
        const float cost = 0.3f * ((col_tiles + parts - 1) / parts) + 1.5f + 0.06f * nt;
        if (cost < least) { least = cost; best = parts; }
    }
    return best;
}
// Shared memory of the quantised rows of a CTA.
u32 raw_bytes(u32 nt, u32 col_tiles, u32 parts, int fmt) {
    return (col_tiles + parts - 1) / parts * nt * (128 + (u32)mx4_pieces(fmt) * 4);
}

// `x`: the few rows as plain values instead of a.p (may be null).
bool launch_narrow(int sms, cudaStream_t s, const Mx4Operand& a, const RowsIn* x, const Mx4Operand& b, u64 cols, int fmt,
                   const Mx4Result& r, u64 wait_ns, u32* flag, bool behind) {
    NarrowArgs g{};
    // b on the M side: neighbouring lanes write neighbouring results
    g.m = b;
    g.n = a;
    g.cols = cols;
    g.col_tiles = mx4_col_tiles(cols);
    g.nt = g.n.rows > MX4_ROWS ? MX4_ROWS : (u32)((g.n.rows + 7) & ~7ull);
    g.n_tiles = mx4_row_tiles(g.n.rows);
    g.y = r.y;
    g.stride = r.stride;
    g.bias = r.bias;
    const u32 sb = (u32)mx4_scale_bytes(fmt), parts = split(sms, mx4_row_tiles(g.m.rows), g.n_tiles, g.nt, g.col_tiles);
    g.stage_bytes = CODES + sb + (x ? 0 : g.nt * 128 + sb);
    u32 smem = g.stage_bytes * STAGES + 1024;
    g.sums = g.stage_bytes * STAGES;
    if (parts > 1) smem += ((g.nt + parts - 1) / parts * parts * MX4_ROWS * 4 + 1023) & ~1023u;      // what follows starts on 1024 bytes
    const u32 need = g.nt + STAGES * (u32)mx4_pieces(fmt) * 8;
    g.tmem_cols = 32;
    while (g.tmem_cols < need) g.tmem_cols *= 2;
    g.early = behind;
    g.wait_ns = wait_ns;
    g.flag = flag;
    if (!x) return launch_typed<-1>(s, g, parts, smem, fmt, r.dtype);
    g.x = x->p;
    g.x_stride = x->stride;
    const u64 size = x->dtype == DT_F32 ? 4 : 2;
    g.x_vec = (reinterpret_cast<uintptr_t>(x->p) & 15) == 0 && (x->rows == 1 || ((x->stride * size) & 15) == 0);
    g.x_codes = smem - 1024;
    g.x_scales = g.x_codes + (g.col_tiles + parts - 1) / parts * g.nt * 128;
    smem += raw_bytes(g.nt, g.col_tiles, parts, fmt);
    return x->dtype == DT_F32 ? launch_typed<DT_F32>(s, g, parts, smem, fmt, r.dtype)
         : x->dtype == DT_F16 ? launch_typed<DT_F16>(s, g, parts, smem, fmt, r.dtype)
                              : launch_typed<DT_BF16>(s, g, parts, smem, fmt, r.dtype);
}

}  // namespace

bool launch_mx4_matmul(int sms, cudaStream_t s, const Mx4Operand& a, const Mx4Operand& b, u64 cols, int fmt,
                       const Mx4Result& r, u64 wait_ns, u32* flag, bool behind) {
    // 256 x 256 tiles only where they are enough for half the pairs of SMs
    const u64 wide_tiles = ((a.rows + 255) / 256) * ((b.rows + 255) / 256);
    if (cols && a.rows > MX4_ROWS && b.rows > MX4_ROWS && wide_tiles * 4 >= (u64)sms)
        return launch_mx4_matmul_wide(sms, s, a, b, cols, fmt, r, wait_ns, flag, behind);
    return launch_narrow(sms, s, a, nullptr, b, cols, fmt, r, wait_ns, flag, behind);
}

bool mx4_linear_in_one(int sms, u64 rows, u64 w_rows, u64 cols) {
    if (rows > RAW_ROWS) return false;
    const u32 nt = (u32)((rows + 7) & ~7ull), ct = mx4_col_tiles(cols), parts = split(sms, mx4_row_tiles(w_rows), 1, nt, ct);
    return rows * ((ct + parts - 1) / parts) <= RAW_TASKS;
}

bool launch_mx4_linear(int sms, cudaStream_t s, const RowsIn& x, const float* x_scale, const Mx4Operand& w, int fmt,
                       const Mx4Result& r, u64 wait_ns, u32* flag) {
    const Mx4Operand a{nullptr, x.rows, x_scale};
    return launch_narrow(sms, s, a, &x, w, x.cols, fmt, r, wait_ns, flag, false);
}

}  // namespace excp
