// The product with plain 16-bit operands: c[i, j] = sum over k of a[i, k] b[j, k], and what is done to it on the way out.
// Shared by the kernels for few rows (product.cu) and for many (product_wide.cu): operands, tensor maps, epilogue.
#pragma once
#include <cuda.h>

#include "layers.cuh"
#include "mx4_pipe.cuh"

namespace excp {

constexpr u32 PR_TILE = 128;                       // rows of an operand tile = lanes of tensor memory
constexpr u32 PR_K = 64;                           // columns of a box: 128 bytes, one swizzle span
// The tensor core cuts its sums off instead of rounding them: 1024 columns added one after the other lose 1e-6 of a sum (measured), 4096
// 4e-6, which shows in a result of 32 bits.  There, and in the kernel for few rows always, the columns are added up in runs of at most so many,
// and the runs' sums in fp32: 7e-7 (of fp16 1e-6) whatever the length, of terms of both signs.  (Runs of 512: 5e-7, and a twelfth slower.)  Where all terms have
// one sign every addition cuts off the same way: of fp16 4e-6, or 6e-9 a column of one run.
constexpr u32 PR_RUN = 768;
// It shows less in fewer bits, and the kernel for many rows takes longer runs for them.
// Codes of 8 bits: after 4096 columns in one run seven times as many as of a plain fp32 sum land on the other side of a border, and the kept values of
// fp16 activations are 1.7 times as far off; runs of 2048 columns leave 1.2 times.  Not shorter with an activation: while such a tile is written out the products
// can go on for two runs only (4096 x 4096 -> 11008, gelu: runs of 768 columns 369 us, of 2048 317).
// (Without one they are as short as for 32 bits, 249 -> 331 us: the result beside 8 bits is then the same as beside 32.)
// Results of 16 bits: the same, so that they do not depend on 8 bits kept beside them.  (One run for all columns is 1.8 us a launch quicker, and fp16
// results of 50304 columns of one sign lost 3e-4 by it, more than half a unit.)
constexpr u32 PR_RUN_16 = 2048;
constexpr u32 PR_CHUNK = 64;                       // rows of a box of an operand that lies the other way round
constexpr u32 PR_CHUNK_BYTES = PR_CHUNK * PR_K * 2;

// One operand: `rows` x `k`.  along_k: its k values are neighbours in memory, rows `stride` apart; else the rows are neighbours
// and k values `stride` apart (a transposed matrix).  On 16 bytes, like its stride.
struct ProductOperand {
    const void* p;
    u64 rows, k, stride;
    bool along_k;
};

// What becomes of a sum v of c[i, j]: p = v + bias[j]; kept = p; y = act(p) + residual[i, j].
struct ProductEnd {
    Matrix y;                                      // rows, cols: of c
    ColumnVector bias;
    int act = ACT_NONE;
    Matrix residual;                               // p null: none
    Matrix kept;                                   // p null: none
};

// Columns of a run of the kernel for many rows.
inline u32 product_run(const ProductEnd& e) {
    const bool kept32 = e.kept.p && e.kept.dtype == DT_F32, kept8 = e.kept.p && e.kept.dtype == DT_ACT8;
    return e.y.dtype == DT_F32 || kept32 || (kept8 && e.act == ACT_NONE) ? PR_RUN : PR_RUN_16;
}

struct ProductCall {
    ProductOperand a, b;
    ProductEnd end;
    int dtype;                                     // of both operands: DT_F16 or DT_BF16
    int device, sms;
    u64 wait_ns;
    u32* flag;
};
bool launch_product(cudaStream_t s, const ProductCall& c);
bool launch_product_wide(cudaStream_t s, const ProductCall& c);
float product_wide_us(const ProductCall& c);       // about how long it takes

// Rows that a tensor map cannot describe (not on 16 bytes) -> rows of `pitch` values in `to`.
u64 tidy_pitch(u64 cols);
void launch_tidy(int sms, cudaStream_t s, const Matrix& m, void* to);

// A map of an operand in boxes of `box_rows` rows (64 where the rows are neighbours) and PR_K columns.
bool product_map(CUtensorMap* map, const ProductOperand& o, u32 box_rows, int dtype);
// A map of a result whose rows start on 16 bytes, in boxes of 32 x 32 (end_rows).
bool result_map(CUtensorMap* map, const Matrix& y);

// The epilogue as the kernels take it.
struct EndArgs {
    void* y;
    u64 stride, rows, cols;
    const void* bias;
    const void* residual;
    u64 residual_stride;
    void* kept;
    u64 kept_stride;
    Kept k8;
    int bias_dtype, act, residual_dtype, kept_dtype;
    // y, kept: rows start on 32 bytes (2), 16 bytes (1) or anywhere (0); residual, bias: on 16 bytes (1)
    u32 y_vec, residual_vec, kept_vec, bias_vec;
};
EndArgs end_args(const ProductEnd& e);

#ifdef __CUDACC__
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, u32 x, u32 y, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Descriptor of an operand tile in shared memory, and what 16 columns further on adds to it.
//   along k   rows of 128 bytes in 128-byte swizzle, eight-row groups 1024 bytes apart; 16 columns are 32 bytes
//   else      boxes of 64 rows (128 bytes) x 64 columns, the same swizzle: eight columns are 1024 bytes, the next 64 rows 8192
__device__ __forceinline__ u64 product_desc(u32 addr, bool along_k) {
    return (u64)((addr >> 4) & 0x3fffu) | ((u64)(along_k ? 1u : PR_CHUNK_BYTES >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ u32 product_desc_step(bool along_k) { return along_k ? 32 >> 4 : 2048 >> 4; }
// fp32 sums, 16-bit operands of one type.
__device__ __forceinline__ u32 product_idesc(bool bf16, bool m_along_k, bool n_along_k, u32 m, u32 n) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (m_along_k ? 0u : 1u << 15) | (n_along_k ? 0u : 1u << 16) | ((n >> 3) << 17) | ((m >> 4) << 24);
}
__device__ __forceinline__ void tm_mma_f16(u32 d, u64 a, u64 b, u32 idesc, u32 add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void tm2_mma_f16(u32 d, u64 a, u64 b, u32 idesc, u32 add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}

// ---- epilogue ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float any_value(const void* p, int dtype, u64 i) {
    if (dtype == DT_F32) return __ldg(static_cast<const float*>(p) + i);
    if (dtype == DT_F16) return __half2float(__ldg(static_cast<const __half*>(p) + i));
    return __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(p) + i));
}
template <u32 W>
__device__ __forceinline__ void activate(float (&f)[W], int act) {
    if (act == ACT_GELU) act_values<ACT_GELU>(f);
    else if (act == ACT_GELU_TANH) act_values<ACT_GELU_TANH>(f);
    else if (act == ACT_SILU) act_values<ACT_SILU>(f);
}
__device__ __forceinline__ void store32(void* p, const u32 v[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// Eight words to a place on 32 bytes (vec = 2) or 16.
__device__ __forceinline__ void store_words(void* p, const u32 (&w)[8], u32 vec) {
    if (vec == 2) {
        store32(p, w);
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
template <typename T>
__device__ __forceinline__ u32 word_of(const float* f) {       // 4 bytes of results
    if constexpr (sizeof(T) == 4) {
        return __float_as_uint(f[0]);
    } else {
        u32 w;
        T* h = reinterpret_cast<T*>(&w);
        wput(h, 0, f[0]);
        wput(h, 1, f[1]);
        return w;
    }
}
// The first `n` of W results to neighbouring places.
template <typename T, u32 W>
__device__ __forceinline__ void put_row(T* y, const float (&f)[W], u32 n, u32 vec) {
    constexpr u32 PER = 4 / sizeof(T), STEP = 8 * PER;
#pragma unroll
    for (u32 i = 0; i < W; i += STEP) {
        if (vec && i + STEP <= n) {
            u32 w[8];
#pragma unroll
            for (u32 k = 0; k < 8; ++k) w[k] = word_of<T>(f + i + k * PER);
            store_words(y + i, w, vec);
        } else {
#pragma unroll
            for (u32 e = i; e < i + STEP; ++e) if (e < n) wput(y, e, f[e]);
        }
    }
}
template <u32 W>
__device__ __forceinline__ void put_row_any(void* p, int dtype, u64 at, const float (&f)[W], u32 n, u32 vec) {
    if (dtype == DT_F32) put_row(static_cast<float*>(p) + at, f, n, vec);
    else if (dtype == DT_F16) put_row(static_cast<__half*>(p) + at, f, n, vec);
    else put_row(static_cast<__nv_bfloat16*>(p) + at, f, n, vec);
}
template <typename T, u32 W>
__device__ __forceinline__ void add_row(const T* r, float (&f)[W], u32 n, bool on16) {
    constexpr u32 PER = 16 / sizeof(T);
#pragma unroll
    for (u32 i = 0; i < W; i += PER) {
        if (on16 && i + PER <= n) {
            const uint4 q = *reinterpret_cast<const uint4*>(r + i);
            const T* h = reinterpret_cast<const T*>(&q);
#pragma unroll
            for (u32 e = 0; e < PER; ++e) f[i + e] += wget(h, e);
        } else {
#pragma unroll
            for (u32 e = i; e < i + PER; ++e) if (e < n) f[e] += wget(r, e);
        }
    }
}

// 32 neighbouring sums of row i, columns j .. j + n - 1: all but the way of y to memory.
__device__ __forceinline__ void end_values(const EndArgs& g, u64 i, u64 j, u32 n, float (&f)[32]) {
    if (g.bias) {
        if (g.bias_dtype == DT_F32) add_row(static_cast<const float*>(g.bias) + j, f, n, g.bias_vec);
        else if (g.bias_dtype == DT_F16) add_row(static_cast<const __half*>(g.bias) + j, f, n, g.bias_vec);
        else add_row(static_cast<const __nv_bfloat16*>(g.bias) + j, f, n, g.bias_vec);
    }
    if (g.kept) {
        if (g.kept_dtype == DT_ACT8) {             // a thread has a whole block of 32
            u32 top = 0;
#pragma unroll
            for (u32 e = 0; e < 32; ++e) {
                if (e >= n) f[e] = 0.f;
                top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
            }
            const float s = a8_scale(top), inverse = a8_inverse(s);
            u32 q[8];
#pragma unroll
            for (u32 k = 0; k < 8; ++k) q[k] = top >= 0x7f800000u ? 0u : a8_codes(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3], inverse);
            const u64 block = i * g.k8.blocks + j / A8_BLOCK;
            store_words(g.k8.codes + block * A8_BLOCK, q, g.kept_vec);
            g.k8.scales[block] = (unsigned short)(__float_as_uint(s) >> 16);
        } else {
            put_row_any(g.kept, g.kept_dtype, i * g.kept_stride + j, f, n, g.kept_vec);
        }
    }
    activate(f, g.act);
    if (g.residual) {
        const u64 at = i * g.residual_stride + j;
        if (g.residual_dtype == DT_F32) add_row(static_cast<const float*>(g.residual) + at, f, n, g.residual_vec);
        else if (g.residual_dtype == DT_F16) add_row(static_cast<const __half*>(g.residual) + at, f, n, g.residual_vec);
        else add_row(static_cast<const __nv_bfloat16*>(g.residual) + at, f, n, g.residual_vec);
    }
}
// The same with y, a lane by itself.
template <int DT>
__device__ __forceinline__ void end_row(const EndArgs& g, u64 i, u64 j, float (&f)[32]) {
    typedef typename ElemOf<DT>::type T;
    if (i >= g.rows || j >= g.cols) return;
    const u32 n = (u32)min((u64)32, g.cols - j);
    end_values(g, i, j, n, f);
    put_row(static_cast<T*>(g.y) + i * g.stride + j, f, n, g.y_vec);
}
// The same of a warp's 32 rows, which a copy takes to memory (rows past the last stay behind; of a row it writes whole 16-byte words, past the
// last column too, so that fewer than 32 columns are left to the lanes).  Lanes that each write 32 bytes of a row of
// their own send 17 bytes a cycle from an SM, whole lines several times that: 16 x 2048 -> 50304, the weight
// gradient in 32 bits: 128 us, so 82.
// `room`: BYTES of shared memory of the warp on 1024 bytes, `turn`: how often it was used.  Before the CTA leaves: end_rows_done.
template <int DT, u32 BYTES>
__device__ __forceinline__ void end_rows(const EndArgs& g, const CUtensorMap* map, unsigned char* room, u32& turn, u64 i, u64 j, float (&f)[32]) {
    typedef typename ElemOf<DT>::type T;
    constexpr u32 LINE = 32 * sizeof(T), BOX = 32 * LINE, ROOMS = BYTES / BOX, PER = 4 / sizeof(T);
    const u32 lane = threadIdx.x & 31;
    if (i - lane >= g.rows || j >= g.cols) return;             // the warp as one
    const u32 n = (u32)min((u64)32, g.cols - j);
    if (i < g.rows) end_values(g, i, j, n, f);
    if (n < 32) {
        if (i < g.rows) put_row(static_cast<T*>(g.y) + i * g.stride + j, f, n, g.y_vec);
        return;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(ROOMS - 1) : "memory");
    __syncwarp();
    unsigned char* to = room + turn++ % ROOMS * BOX;
    const u32 turned = LINE == 128 ? lane & 7 : lane >> 1 & 3; // the swizzle of a row's 16-byte words
#pragma unroll
    for (u32 c = 0; c < LINE / 16; ++c)
        *reinterpret_cast<uint4*>(to + lane * LINE + ((c ^ turned) << 4)) =
            make_uint4(word_of<T>(f + c * 4 * PER), word_of<T>(f + (c * 4 + 1) * PER), word_of<T>(f + (c * 4 + 2) * PER), word_of<T>(f + (c * 4 + 3) * PER));
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // the copy reads what was just written
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
                     ::"l"(map), "r"((u32)j), "r"((u32)i), "r"(smem_u32(to)) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    __syncwarp();
}
__device__ __forceinline__ void end_rows_done() {
    if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
}

// The bias of a column, for end_column.
__device__ __forceinline__ float column_bias(const EndArgs& g, u64 j) { return g.bias && j < g.cols ? any_value(g.bias, g.bias_dtype, j) : 0.f; }

template <typename T, u32 W, bool FULL>
__device__ __forceinline__ void put_column(T* y, u64 stride, u32 n, const float (&f)[W]) {
#pragma unroll
    for (u32 e = 0; e < W; ++e) {
        if (FULL || e < n) wput(y, 0, f[e]);
        y += stride;
    }
}
// Not through the read-only cache: y may be the residual.
template <typename T, u32 W, bool FULL>
__device__ __forceinline__ void add_column(const T* r, u64 stride, u32 n, float (&f)[W]) {
    float v[W];
#pragma unroll
    for (u32 e = 0; e < W; ++e) {
        v[e] = FULL || e < n ? wget(r, 0) : 0.f;
        r += stride;
    }
#pragma unroll
    for (u32 e = 0; e < W; ++e) f[e] += v[e];
}

// W sums of column j (a lane has one; the lanes of a warp have neighbouring ones, the first a multiple of 32), rows i .. i + n - 1.
template <int DT, u32 W, bool FULL>
__device__ __forceinline__ void end_column_of(const EndArgs& g, u64 i, u64 j, u32 n, float bias, float (&f)[W]) {
    typedef typename ElemOf<DT>::type T;
    const bool there = j < g.cols;
    if (g.bias) {
#pragma unroll
        for (u32 e = 0; e < W; ++e) f[e] += bias;
    }
    if (g.kept && g.kept_dtype == DT_ACT8) {       // a block is the warp's 32 columns
        const u32 lane = threadIdx.x & 31;
        const u64 block = j / A8_BLOCK;
        if (block < g.k8.blocks) {
            const u64 at = i * g.k8.blocks + block;
            unsigned char* codes = g.k8.codes + at * A8_BLOCK + lane;
            unsigned short* scales = g.k8.scales + at;
#pragma unroll
            for (u32 e = 0; e < W; ++e) {
                const float v = there && (FULL || e < n) ? f[e] : 0.f;
                const u32 top = __reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu);
                const float s = a8_scale(top);
                if (FULL || e < n) {
                    *codes = top >= 0x7f800000u ? 0 : (unsigned char)a8_codes(v, 0.f, 0.f, 0.f, a8_inverse(s));
                    if (lane == 0) *scales = (unsigned short)(__float_as_uint(s) >> 16);
                }
                codes += g.k8.blocks * A8_BLOCK;
                scales += g.k8.blocks;
            }
        }
    }
    if (!there) return;
    if (g.kept && g.kept_dtype != DT_ACT8) {
        const u64 at = i * g.kept_stride + j;
        if (g.kept_dtype == DT_F32) put_column<float, W, FULL>(static_cast<float*>(g.kept) + at, g.kept_stride, n, f);
        else if (g.kept_dtype == DT_F16) put_column<__half, W, FULL>(static_cast<__half*>(g.kept) + at, g.kept_stride, n, f);
        else put_column<__nv_bfloat16, W, FULL>(static_cast<__nv_bfloat16*>(g.kept) + at, g.kept_stride, n, f);
    }
    activate(f, g.act);
    if (g.residual) {
        const u64 at = i * g.residual_stride + j;
        if (g.residual_dtype == DT_F32) add_column<float, W, FULL>(static_cast<const float*>(g.residual) + at, g.residual_stride, n, f);
        else if (g.residual_dtype == DT_F16) add_column<__half, W, FULL>(static_cast<const __half*>(g.residual) + at, g.residual_stride, n, f);
        else add_column<__nv_bfloat16, W, FULL>(static_cast<const __nv_bfloat16*>(g.residual) + at, g.residual_stride, n, f);
    }
    put_column<T, W, FULL>(static_cast<T*>(g.y) + i * g.stride + j, g.stride, n, f);
}
template <int DT, u32 W>
__device__ __forceinline__ void end_column(const EndArgs& g, u64 i, u64 j, u32 n, float bias, float (&f)[W]) {
    if (n >= W) end_column_of<DT, W, true>(g, i, j, W, bias, f);
    else end_column_of<DT, W, false>(g, i, j, n, bias, f);
}
#endif

}  // namespace excp
