// The layers before the logits and the way back through them: norms, activations kept in 8 bits, products with plain weights.
// Shared declarations: operands, the packed 8-bit layout, how a row is dealt to threads, column sums, launch wrappers.
#pragma once
#include <type_traits>

#include "activation.cuh"
#include "score_launch.cuh"

namespace excp {

constexpr int DT_ACT8 = 3;                         // a matrix in 8 bits (include/excp.h)

// A matrix in ordinary layout, or in 8 bits (p: the packed buffer; the stride is not looked at).  p null: absent.
struct Matrix {
    void* p = nullptr;
    int dtype = DT_F32;
    u64 rows = 0, cols = 0, stride = 0;
};
// One value per column, of type `dtype`; p null: absent.
struct ColumnVector {
    const void* p = nullptr;
    int dtype = DT_F32;
};

// ---- 8 bits: rows of 32 ceil(C / 32) signed bytes, then rows of ceil(C / 32) bfloat16 scales -----------------------------
constexpr u32 A8_BLOCK = 32;
__host__ __device__ inline u64 a8_blocks(u64 cols) { return (cols + A8_BLOCK - 1) / A8_BLOCK; }
__host__ __device__ inline u64 a8_bytes(u64 rows, u64 cols) { return (rows * a8_blocks(cols) * (A8_BLOCK + 2) + 15) & ~15ull; }

// ---- launch wrappers ---------------------------------------------------------------------------------------------------
void launch_act8_quantize(int sms, cudaStream_t s, const Matrix& x, unsigned char* packed);
void launch_act8_restore(int sms, cudaStream_t s, const unsigned char* packed, const Matrix& out);

u64 act_grad_scratch(int sms, u64 rows, u64 cols);
void launch_act_grad(int sms, cudaStream_t s, int act, const Matrix& dy, const Matrix& pre, const Matrix& dpre, const Matrix& again, float* dbias,
                     float* scratch);

void launch_layer_norm(int sms, cudaStream_t s, const Matrix& x, const ColumnVector& weight, const ColumnVector& bias, float eps, bool rms,
                       const Matrix& y, float* row_stats, unsigned char* kept);
u64 layer_norm_grad_scratch(int sms, u64 rows, u64 cols);
void launch_layer_norm_grad(int sms, cudaStream_t s, const Matrix& dy, const Matrix& x, const ColumnVector& weight, bool rms, const float* row_stats,
                            const Matrix& add, const Matrix& dx, float* dweight, float* dbias, float* scratch);

// Sums over `parts` rows of `n` floats each, in the order of the rows: out0 gets the first `split` columns, out1 the rest (null: not
// wanted).
void launch_column_sums(cudaStream_t s, const float* rows, u32 parts, u64 n, u64 split, float* out0, float* out1);

#ifdef __CUDACC__
// ---- how a warp holds 256 consecutive columns of a row, eight to a lane -------------------------------------------------
// VEC: eight neighbours, fetched in 16-byte words (rows on 16 bytes).  Else column 32 e + lane for e = 0 .. 7, so that the lanes of
// one access are neighbours whatever the alignment.  Either way 32 lanes x 8 values are eight whole blocks of an 8-bit matrix.
template <bool VEC>
__device__ __forceinline__ u32 lane_col(u32 base, u32 lane, u32 e) {
    return VEC ? base + lane * 8 + e : base + e * 32 + lane;
}

// Sixteen bytes of values as they lie in memory, and as fp32.
template <typename T, bool VEC>
struct Raw {
    static constexpr int N = VEC ? (int)sizeof(T) / 2 : 8;
    typename std::conditional<VEC, uint4, T>::type q[N];

    // Columns past `cols` are left 0.
    __device__ __forceinline__ void load(const T* row, u32 base, u32 lane, u32 cols) {
        if constexpr (VEC) {
            const u32 c = base + lane * 8;
            if (c + 8 <= cols) {
                const uint4* p = reinterpret_cast<const uint4*>(row + c);
#pragma unroll
                for (int i = 0; i < N; ++i) q[i] = __ldg(p + i);
            } else {
                T* h = reinterpret_cast<T*>(q);
#pragma unroll
                for (int e = 0; e < 8; ++e) wput(h, e, c + e < cols ? wget(row, c + e) : 0.f);
            }
        } else {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) {
                const u32 c = base + e * 32 + lane;
                if (c < cols) q[e] = row[c];
                else wput(q, e, 0.f);
            }
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        const T* h = reinterpret_cast<const T*>(q);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = wget(h, e);
    }
};

template <typename T, bool VEC>
__device__ __forceinline__ void load_cols(const T* row, u32 base, u32 lane, u32 cols, float (&v)[8]) {
    Raw<T, VEC> r;
    r.load(row, base, lane, cols);
    r.values(v);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_cols(T* row, u32 base, u32 lane, u32 cols, const float (&v)[8]) {
    if constexpr (VEC) {
        const u32 c = base + lane * 8;
        if (c + 8 <= cols) {
            uint4 q[sizeof(T) / 2];
            T* h = reinterpret_cast<T*>(q);
#pragma unroll
            for (int e = 0; e < 8; ++e) wput(h, e, v[e]);
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) __stcs(reinterpret_cast<uint4*>(row + c) + i, q[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < cols) wput(row, c + e, v[e]);
        }
    } else {
#pragma unroll
        for (u32 e = 0; e < 8; ++e) {
            const u32 c = base + e * 32 + lane;
            if (c < cols) wput(row, c, v[e]);
        }
    }
}
// One value per column, 32-bit floats or T (runtime: the branch is the same for all).
template <typename T, bool VEC>
__device__ __forceinline__ void load_vector(const ColumnVector& w, u32 base, u32 lane, u32 cols, float absent, float (&v)[8]) {
    if (!w.p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = absent;
    } else if (w.dtype == DT_F32) {
        load_cols<float, VEC>(static_cast<const float*>(w.p), base, lane, cols, v);
    } else {
        load_cols<T, VEC>(static_cast<const T*>(w.p), base, lane, cols, v);
    }
}

// ---- blocks of 32 values in 8 bits ------------------------------------------------------------------------------------------
// The scale of a block from its largest magnitude (as bits): A / 127 rounded up to 8 significant bits, at least 2^-126; NaN where the
// block holds one or an infinity.  It has the bits of a bfloat16.
__device__ __forceinline__ float a8_scale(u32 largest) {
    if (largest >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const u32 b = (__float_as_uint(__fdiv_rn(__uint_as_float(largest), 127.f)) + 0xffffu) & 0xffff0000u;
    return __uint_as_float(max(b, 0x00800000u));
}
// Four codes in a word.  1.5 * 2^23 added: the nearest whole number (ties to even) in the low byte, in two's complement.
__device__ __forceinline__ u32 a8_codes(float a, float b, float c, float d, float inverse) {
    constexpr float M = 12582912.f;
    const u32 ab = __byte_perm(__float_as_uint(a * inverse + M), __float_as_uint(b * inverse + M), 0x0040);
    const u32 cd = __byte_perm(__float_as_uint(c * inverse + M), __float_as_uint(d * inverse + M), 0x0040);
    return __byte_perm(ab, cd, 0x5410);
}
// 1 / scale; of NaN: 0 where that makes every code 0.
__device__ __forceinline__ float a8_inverse(float scale) { return __frcp_rn(scale); }
// The value of byte `i` of a word of codes that was turned to 0 .. 255 (^ 0x80808080).
__device__ __forceinline__ float a8_value(u32 turned, u32 i, float scale) {
    return (__uint_as_float(__byte_perm(turned, 0x4b000000u, 0x7440u + i)) - 8388736.f) * scale;
}

struct Kept {                                      // an 8-bit matrix
    unsigned char* codes = nullptr;
    unsigned short* scales = nullptr;
    u32 blocks = 0;                                // per row
    Kept() = default;
    __host__ __device__ __forceinline__ Kept(void* p, u64 rows, u64 cols)
        : codes(static_cast<unsigned char*>(p)), scales(reinterpret_cast<unsigned short*>(static_cast<unsigned char*>(p) + rows * a8_blocks(cols) * A8_BLOCK)),
          blocks((u32)a8_blocks(cols)) {}
};

// The lane's eight values -> codes and scales.  Whole warp; values past `cols` are 0.
template <bool VEC>
__device__ __forceinline__ void store_kept(const Kept& k, u64 row, u32 base, u32 lane, u32 cols, const float (&v)[8]) {
    unsigned char* codes = k.codes + row * k.blocks * A8_BLOCK;
    unsigned short* scales = k.scales + row * k.blocks;
    if constexpr (VEC) {
        u32 top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float s = a8_scale(top), inverse = a8_inverse(s);
        uint2 q = make_uint2(a8_codes(v[0], v[1], v[2], v[3], inverse), a8_codes(v[4], v[5], v[6], v[7], inverse));
        if (top >= 0x7f800000u) q = make_uint2(0u, 0u);
        const u32 c = base + lane * 8;
        if (c / A8_BLOCK < k.blocks) {
            *reinterpret_cast<uint2*>(codes + c) = q;
            if ((lane & 3) == 0) scales[c / A8_BLOCK] = (unsigned short)(__float_as_uint(s) >> 16);
        }
    } else {
#pragma unroll
        for (u32 e = 0; e < 8; ++e) {
            const u32 b = base / A8_BLOCK + e;
            if (b >= k.blocks) break;
            const u32 top = __reduce_max_sync(0xffffffffu, __float_as_uint(v[e]) & 0x7fffffffu);
            const float s = a8_scale(top);
            const u32 q = top >= 0x7f800000u ? 0u : a8_codes(v[e], 0.f, 0.f, 0.f, a8_inverse(s));
            codes[b * A8_BLOCK + lane] = (unsigned char)q;
            if (lane == 0) scales[b] = (unsigned short)(__float_as_uint(s) >> 16);
        }
    }
}

template <bool VEC>
struct RawKept {                                   // a lane's eight codes and their scales as they lie in memory
    u32 q[VEC ? 2 : 8];
    unsigned short s[VEC ? 1 : 8];
    __device__ __forceinline__ void load(const Kept& k, u64 row, u32 base, u32 lane, u32) {
        const unsigned char* codes = k.codes + row * k.blocks * A8_BLOCK;
        const unsigned short* scales = k.scales + row * k.blocks;
        if constexpr (VEC) {
            const u32 c = base + lane * 8;
            const bool there = c / A8_BLOCK < k.blocks;
            const uint2 w = there ? __ldg(reinterpret_cast<const uint2*>(codes + c)) : make_uint2(0u, 0u);
            q[0] = w.x;
            q[1] = w.y;
            s[0] = there ? __ldg(scales + c / A8_BLOCK) : 0;
        } else {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) {
                const u32 b = base / A8_BLOCK + e;
                q[e] = b < k.blocks ? codes[b * A8_BLOCK + lane] : 0u;
                s[e] = b < k.blocks ? scales[b] : 0;
            }
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if constexpr (VEC) {
            const float scale = __uint_as_float((u32)s[0] << 16);
#pragma unroll
            for (u32 e = 0; e < 8; ++e) v[e] = a8_value(q[e / 4] ^ 0x80808080u, e % 4, scale);
        } else {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) v[e] = a8_value(q[e] ^ 0x80u, 0, __uint_as_float((u32)s[e] << 16));
        }
    }
};
#endif

}  // namespace excp
