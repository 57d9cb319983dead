// The product with plain 16-bit operands: c[i, j] = sum over k of a[i, k] b[j, k], fp32 sums, and its epilogue.
// This file: few rows on one side (the tokens of a decoding step), or too few tiles for the kernel of many (product_wide.cu).
//
// Bound: with few rows the bytes of the larger operand.  Its rows go on the M side of the tensor core (128 per tile), the few rows on the
// N side, which takes them in steps of 16.  Two CTAs share an SM, and the columns of a tile are split over a cluster so that
// every SM streams; each CTA sends its part of a column of the accumulator to the CTA that owns the column (distributed
// shared memory), which adds them in a fixed order.
//
// Roles: warp 4 fetches both operands (tensor maps; what lies past an edge comes as 0), warp 5 issues the products, warps 0..3
// write the result.
// Every wait for a copy or a product is bounded; where one runs out the CTA raises the handle's flag, lets its copies land and
// leaves.  The two that hardware gives no limit, for tensor memory and at the cluster's barrier, depend only on CTAs whose own
// waits are bounded.
#include "product.cuh"

namespace excp {
namespace {

constexpr int WORK_WARPS = 4;
constexpr u32 FETCH_WARP = WORK_WARPS, PRODUCT_WARP = WORK_WARPS + 1;
constexpr int THREADS = (WORK_WARPS + 2) * 32;
constexpr int STAGES_MAX = 12;
constexpr u32 MAX_SPLIT = 8;
constexpr u32 M_BYTES = PR_TILE * PR_K * 2;
constexpr u32 SMEM_MAX = 227 * 1024 - 1024;        // dynamic shared memory of a block, beside what the kernel has of its own

struct NarrowArgs {
    CUtensorMap m, n;
    u32 m_along_k, n_along_k, bf16;
    u32 k_tiles, n_tiles;
    u32 nt;                                        // rows of n per CTA: a multiple of 16, at most 256
    u32 n_bytes, stages, tmem_cols;
    u32 per_owner;                                 // columns of the accumulator that a CTA of the cluster joins
    u32 turned;                                    // m is b: a lane has a column of c
    EndArgs end;
    u64 wait_ns;
    u32* flag;
};

struct Shared {
    unsigned long long full[STAGES_MAX];           // copies have landed
    unsigned long long empty[STAGES_MAX];          // the stage has been multiplied
    unsigned long long done;
    u32 tmem;
    volatile u32 abort;
};

struct Turn {                                      // the place in the ring of stages, and the parity of its current turn
    u32 s = 0, parity = 0;
    __device__ __forceinline__ void next(u32 stages) {
        if (++s == stages) { s = 0; parity ^= 1; }
    }
};

template <int DT>
__global__ void __launch_bounds__(THREADS, 2) product_kernel(const __grid_constant__ NarrowArgs g) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ Shared sh;
    const u32 part = cluster_rank(), parts = cluster_size();
    // the swizzle goes by address: stages start on 1024 bytes (the same offset in every CTA)
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const u32 warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const u32 tile = blockIdx.x / parts, mt = tile / g.n_tiles, ntile = tile - mt * g.n_tiles;
    const u32 k0 = (u32)((u64)g.k_tiles * part / parts), k1 = (u32)((u64)g.k_tiles * (part + 1) / parts);
    const u32 stage = M_BYTES + g.n_bytes;
    float* const joined = reinterpret_cast<float*>(smem + g.stages * stage);       // [part][own column][row]

    if (threadIdx.x == 0) {
        for (u32 s = 0; s < g.stages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        mbar_init(&sh.done, 1);
        sh.abort = 0;
        mbar_fence_init();
    }
    if (warp == PRODUCT_WARP) tm_alloc(&sh.tmem, g.tmem_cols);
    if (warp == FETCH_WARP && g.k_tiles && elect_one()) { tma_prefetch_map(&g.m); tma_prefetch_map(&g.n); }
    __syncwarp();
    wait_for_previous();
    let_next_start();
    tm_fence_before();
    __syncthreads();
    if (parts > 1) cluster_arrive();
    tm_fence_after();
    const u32 tmem = sh.tmem;
    bool ok = true;                                // this warp's waits were all met

    if (warp == FETCH_WARP) {
        Turn ring;
        u32 filled = 0;
        const u32 m_row = mt * PR_TILE, n_row = ntile * g.nt;
        for (u32 k = k0; k < k1; ++k) {
            if (filled >= g.stages && !(ok = wait_warp(&sh, &sh.empty[ring.s], ring.parity ^ 1, g.wait_ns, g.flag))) break;
            unsigned char* st = smem + ring.s * stage;
            unsigned long long* bar = &sh.full[ring.s];
            if (elect_one()) {
                mbar_arrive_expect_tx(bar, stage);
                if (g.m_along_k) {
                    tma_load_2d(st, &g.m, k * PR_K, m_row, bar);
                } else {
                    tma_load_2d(st, &g.m, m_row, k * PR_K, bar);
                    tma_load_2d(st + PR_CHUNK_BYTES, &g.m, m_row + PR_CHUNK, k * PR_K, bar);
                }
                if (g.n_along_k) tma_load_2d(st + M_BYTES, &g.n, k * PR_K, n_row, bar);
                else for (u32 c = 0; c < g.nt; c += PR_CHUNK) tma_load_2d(st + M_BYTES + c / PR_CHUNK * PR_CHUNK_BYTES, &g.n, n_row + c, k * PR_K, bar);
            }
            __syncwarp();
            ++filled;
            ring.next(g.stages);
        }
        // no copy may be in flight when the CTA leaves: the last turn of every stage that was filled
        for (u32 i = 0; i < g.stages && i < filled; ++i) {
            if (ring.s == 0) { ring.s = g.stages; ring.parity ^= 1; }
            --ring.s;
            drain_warp(&sh.full[ring.s], ring.parity);
        }
    } else if (warp == PRODUCT_WARP) {
        const u32 idesc = product_idesc(g.bf16, g.m_along_k, g.n_along_k, PR_TILE, g.nt);
        const u32 step_m = product_desc_step(g.m_along_k), step_n = product_desc_step(g.n_along_k);
        Turn ring;
        for (u32 k = k0; k < k1; ++k) {
            if (!(ok = wait_warp(&sh, &sh.full[ring.s], ring.parity, g.wait_ns, g.flag))) break;
            tm_fence_after();
            const u32 st = smem_u32(smem) + ring.s * stage;
            const u64 dm = product_desc(st, g.m_along_k), dn = product_desc(st + M_BYTES, g.n_along_k);
            if (elect_one()) {
#pragma unroll
                for (u32 i = 0; i < PR_K / 16; ++i) tm_mma_f16(tmem, dm + i * step_m, dn + i * step_n, idesc, k > k0 || i);
                tm_commit(&sh.empty[ring.s]);
            }
            __syncwarp();
            ring.next(g.stages);
        }
        if (elect_one()) tm_commit(&sh.done);
        __syncwarp();
        drain_warp(&sh.done, 0);                   // what has been issued is done before tensor memory goes
    } else {
        ok = wait_warp(&sh, &sh.done, 0, g.wait_ns, g.flag);
        tm_fence_after();
    }

    const u32 t = threadIdx.x;
    const u64 m = (u64)mt * PR_TILE + t, n0 = (u64)ntile * g.nt, n_rows = g.turned ? g.end.rows : g.end.cols;
    const u32 cols = (u32)min((u64)g.nt, n_rows - n0);         // of the accumulator that are results
    // Columns c .. c + W - 1 of the accumulator, complete.  Whole warps.
    auto put = [&](auto width, u32 c, float (&f)[decltype(width)::value]) {
        constexpr u32 W = decltype(width)::value;
        if (c >= cols) return;
        if (g.turned) end_column<DT, W>(g.end, n0 + c, m, min(W, cols - c), f);
        else if constexpr (W == 32) end_row<DT>(g.end, m, n0 + c, f);
    };
    auto take = [&](auto width, u32 c) {
        constexpr u32 W = decltype(width)::value;
        u32 v[W];
        __syncwarp();
        if constexpr (W == 32) tm_load32(tmem + ((warp * 32) << 16) + c, v);
        else { tm_load8(tmem + ((warp * 32) << 16) + c, v); tm_load8(tmem + ((warp * 32) << 16) + c + 8, v + 8); }
        tm_wait_load();
        float f[W];
#pragma unroll
        for (u32 e = 0; e < W; ++e) f[e] = k0 < k1 ? __uint_as_float(v[e]) : 0.f;
        if (parts == 1) {
            put(width, c, f);
        } else {
            // column c belongs to CTA c / per_owner, which has a place for this CTA's part of it
            u32 owner = c / g.per_owner, place = c - owner * g.per_owner;
#pragma unroll
            for (u32 e = 0; e < W; ++e) {
                if (c + e < cols) st_cluster(cluster_address(joined + (part * g.per_owner + place) * PR_TILE + t, owner), f[e]);
                if (++place == g.per_owner) { place = 0; ++owner; }
            }
        }
    };
    if (parts > 1) cluster_wait();                 // every CTA of the cluster has started
    if (warp < WORK_WARPS) {
        if (g.nt >= 32) {
            for (u32 c = 0; c < cols; c += 32) take(std::integral_constant<u32, 32>(), c);
        } else {
            take(std::integral_constant<u32, 16>(), 0);
        }
        tm_fence_before();
    }
    __syncwarp();
    if (parts > 1) {
        cluster_arrive_release();
        cluster_wait();
        if (warp < WORK_WARPS) {
            const u32 first = part * g.per_owner, count = first < cols ? min(g.per_owner, cols - first) : 0;
            auto join = [&](auto width, u32 c) {   // own columns c ..: their parts in ascending order
                constexpr u32 W = decltype(width)::value;
                float f[W];
#pragma unroll
                for (u32 e = 0; e < W; ++e) f[e] = joined[min(c + e, g.per_owner - 1) * PR_TILE + t];
                for (u32 p = 1; p < parts; ++p) {
#pragma unroll
                    for (u32 e = 0; e < W; ++e) f[e] += joined[(p * g.per_owner + min(c + e, g.per_owner - 1)) * PR_TILE + t];
                }
                if (g.turned) end_column<DT, W>(g.end, n0 + first + c, m, min(W, count - c), f);
                else if constexpr (W == 32) end_row<DT>(g.end, m, n0 + first + c, f);
            };
            if (!g.turned) for (u32 c = 0; c < count; c += 32) join(std::integral_constant<u32, 32>(), c);
            else for (u32 c = 0; c < count; c += 8) join(std::integral_constant<u32, 8>(), c);
        }
    }
    __syncwarp();
    __syncthreads();
    tm_fence_after();
    if (warp == PRODUCT_WARP) tm_dealloc(tmem, g.tmem_cols);
}

template <int DT>
bool launch_as(cudaStream_t s, const NarrowArgs& g, u32 blocks, u32 parts, u32 smem) {
    static std::atomic<u64> allowed{0};
    if (!allow_smem(product_kernel<DT>, allowed, SMEM_MAX)) return false;
    return launch_chained(product_kernel<DT>, blocks, THREADS, smem, parts, s, g);
}

bool launch_narrow(cudaStream_t s, const ProductCall& c) {
    NarrowArgs g;
    g.end = end_args(c.end);
    // The fewer rows on the N side: b's rows on the M side where that leaves fewer tiles, or rows of y do not start on 32 bytes.
    const bool few_a = c.a.rows <= c.b.rows;
    const u64 few = few_a ? c.a.rows : c.b.rows;
    g.turned = few <= PR_TILE ? few_a : !g.end.y_vec;
    const ProductOperand& m = g.turned ? c.b : c.a;
    const ProductOperand& n = g.turned ? c.a : c.b;
    g.nt = n.rows >= PR_TILE ? PR_TILE : (u32)((n.rows + 15) & ~15ull);
    if (!g.turned && g.nt < PR_TILE) g.nt = (g.nt + 31) & ~31u;        // whole blocks of 32 columns
    g.n_tiles = (u32)((n.rows + g.nt - 1) / g.nt);
    g.k_tiles = (u32)((m.k + PR_K - 1) / PR_K);
    const u64 m_tiles = (m.rows + PR_TILE - 1) / PR_TILE;
    u32 parts = 1;
    while (parts < MAX_SPLIT && m_tiles * g.n_tiles * (parts + 1) <= (u64)c.sms * 2 && g.k_tiles >= 4 * (parts + 1)) ++parts;
    g.n_bytes = n.along_k ? g.nt * PR_K * 2 : (g.nt + PR_CHUNK - 1) / PR_CHUNK * PR_CHUNK_BYTES;
    g.per_owner = (g.nt + parts - 1) / parts;
    if (!g.turned) g.per_owner = (g.per_owner + 31) & ~31u;
    const u32 sums = parts > 1 ? parts * g.per_owner * PR_TILE * 4 : 0, stage = M_BYTES + g.n_bytes;
    const u32 room = SMEM_MAX / 2 - 1024 - 1024;   // two CTAs to an SM
    u32 stages = (room > sums ? room - sums : 0) / stage;
    if (stages < 3) stages = (SMEM_MAX - 1024 - sums) / stage;
    if (stages > STAGES_MAX) stages = STAGES_MAX;
    if (stages > (g.k_tiles + parts - 1) / parts) stages = (g.k_tiles + parts - 1) / parts;
    g.stages = stages ? stages : 1;
    g.tmem_cols = 32;
    while (g.tmem_cols < g.nt) g.tmem_cols *= 2;
    if (g.k_tiles && (!product_map(&g.m, m, PR_TILE, c.dtype) || !product_map(&g.n, n, g.nt, c.dtype))) return false;
    g.m_along_k = m.along_k;
    g.n_along_k = n.along_k;
    g.bf16 = c.dtype == DT_BF16;
    g.wait_ns = c.wait_ns;
    g.flag = c.flag;
    const u32 smem = g.stages * stage + sums + 1024, blocks = (u32)(m_tiles * g.n_tiles) * parts;
    return c.end.y.dtype == DT_F32 ? launch_as<DT_F32>(s, g, blocks, parts, smem)
         : c.end.y.dtype == DT_F16 ? launch_as<DT_F16>(s, g, blocks, parts, smem)
                                   : launch_as<DT_BF16>(s, g, blocks, parts, smem);
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

bool product_map(CUtensorMap* map, const ProductOperand& o, u32 box_rows, int dtype) {
    static const auto encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(f);
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {o.along_k ? o.k : o.rows, o.along_k ? o.rows : o.k}, strides[1] = {o.stride * 2};
    const cuuint32_t box[2] = {PR_K, o.along_k ? box_rows : PR_K}, one[2] = {1, 1};
    return encode(map, dtype == DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(o.p), dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
    g.y_vec = on(e.y, 32);
    g.residual_vec = e.residual.p && on(e.residual, 16);
    g.kept_vec = e.kept.p && (e.kept.dtype == DT_ACT8 ? (reinterpret_cast<uintptr_t>(e.kept.p) & 31) == 0 : on(e.kept, 32));
    return g;
}

bool launch_product(cudaStream_t s, const ProductCall& c) {
    // 256 x 256 tiles only where they are enough for half the pairs of SMs
    const u64 wide_tiles = ((c.a.rows + 255) / 256) * ((c.b.rows + 255) / 256);
    if (c.a.k && c.a.rows > PR_TILE && c.b.rows > PR_TILE && wide_tiles * 4 >= (u64)c.sms) return launch_product_wide(s, c);
    return launch_narrow(s, c);
}

}  // namespace excp
