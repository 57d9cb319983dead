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

// Whether a kernel may take a matrix (or vector) in 16-byte words.
inline bool on_words(const void* p, u64 stride_bytes, u64 rows) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows == 1 || (stride_bytes & 15) == 0); }
inline bool in_words(const Matrix& m) { return !m.p || (m.cols % 8 == 0 && (m.dtype == DT_ACT8 || on_words(m.p, m.stride * (m.dtype == DT_F32 ? 4 : 2), m.rows))); }
inline bool in_words(const ColumnVector& v) { return on_words(v.p, 0, 1); }

// ---- launch wrappers ---------------------------------------------------------------------------------------------------
void launch_act8_quantize(cudaStream_t s, const Matrix& x, unsigned char* packed);
void launch_act8_restore(cudaStream_t s, const unsigned char* packed, const Matrix& out);

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
// VEC: eight neighbours, fetched in 16-byte words (rows on 16 bytes, of a multiple of eight columns: an edge inside a word would double the
// code of every piece, and these kernels wait for instructions before they wait for memory).  Else column 32 e + lane for e = 0 .. 7, so that the lanes of
// one access are neighbours whatever the alignment.  Either way 32 lanes x 8 values are eight whole blocks of an 8-bit matrix.
template <bool VEC>
__device__ __forceinline__ u32 lane_col(u32 base, u32 lane, u32 e) {
    return VEC ? base + lane * 8 + e : base + e * 32 + lane;
}

// A lane's eight values, two to a word: neighbours (VEC), or those of columns 32 e + lane and 32 (e + 1) + lane.
typedef f32x2 Eight[4];

template <typename T> __device__ __forceinline__ f32x2 two_values(const void* p);          // of a 4-byte word (fp32: of 8 bytes)
template <> __device__ __forceinline__ f32x2 two_values<float>(const void* p) { return *static_cast<const f32x2*>(p); }
template <> __device__ __forceinline__ f32x2 two_values<__half>(const void* p) {
    const float2 f = __half22float2(*static_cast<const __half2*>(p));
    return pack_2(f.x, f.y);
}
template <> __device__ __forceinline__ f32x2 two_values<__nv_bfloat16>(const void* p) {
    const u32 w = *static_cast<const u32*>(p);
    return (u64)(w << 16) | (u64)(w & 0xffff0000u) << 32;
}
template <typename T>
__device__ __forceinline__ void put_two(void* p, f32x2 v) {
    if constexpr (sizeof(T) == 4) *static_cast<f32x2*>(p) = v;
    else if constexpr (std::is_same<T, __half>::value) *static_cast<__half2*>(p) = __floats2half2_rn(low_2(v), high_2(v));
    else *static_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(low_2(v), high_2(v));
}

__device__ __forceinline__ uint4 load_once(const uint4* p) {
    uint4 q;
    asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}

// Eight values as they lie in memory, and as fp32.
template <typename T, bool VEC>
struct Raw {
    static constexpr int N = VEC ? (int)sizeof(T) / 2 : 8;
    typename std::conditional<VEC, uint4, T>::type q[N];

    // Columns past `cols` are left 0.  STREAM: read once (it leaves the first-level cache to what every row reads).
    template <bool STREAM = true>
    __device__ __forceinline__ void load(const T* row, u32 base, u32 lane, u32 cols) {
        if constexpr (VEC) {
            const u32 c = base + lane * 8;
            const uint4* p = reinterpret_cast<const uint4*>(row + c);
#pragma unroll
            for (int i = 0; i < N; ++i) q[i] = c < cols ? (STREAM ? load_once(p + i) : __ldg(p + i)) : make_uint4(0u, 0u, 0u, 0u);
        } else {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) {
                const u32 c = base + e * 32 + lane;
                if (c < cols) q[e] = row[c];
                else wput(q, e, 0.f);
            }
        }
    }
    // VEC: eight at p, or 0.
    template <bool STREAM = true>
    __device__ __forceinline__ void load_at(const T* p, bool there) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint4* w = reinterpret_cast<const uint4*>(p) + i;
            q[i] = there ? (STREAM ? load_once(w) : __ldg(w)) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    __device__ __forceinline__ void values(Eight& v) const {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = two_values<T>(reinterpret_cast<const char*>(q) + i * 2 * sizeof(T));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pack_2(wget(q, 2 * i), wget(q, 2 * i + 1));
        }
    }
};

template <typename T, bool VEC, bool STREAM = true>
__device__ __forceinline__ void load_cols(const T* row, u32 base, u32 lane, u32 cols, Eight& v) {
    Raw<T, VEC> r;
    r.template load<STREAM>(row, base, lane, cols);
    r.values(v);
}
template <typename T>
__device__ __forceinline__ void store_eight(T* p, const Eight& v) {
    uint4 q[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < 4; ++i) put_two<T>(reinterpret_cast<char*>(q) + i * 2 * sizeof(T), v[i]);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) __stcs(reinterpret_cast<uint4*>(p) + i, q[i]);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_cols(T* row, u32 base, u32 lane, u32 cols, const Eight& v) {
    if constexpr (VEC) {
        const u32 c = base + lane * 8;
        if (c < cols) store_eight(row + c, v);
    } else {
#pragma unroll
        for (u32 e = 0; e < 8; ++e) {
            const u32 c = base + e * 32 + lane;
            if (c < cols) wput(row, c, e % 2 ? high_2(v[e / 2]) : low_2(v[e / 2]));
        }
    }
}
// v for the pair i of a lane's eight columns, 0 past the last one.
template <bool VEC>
__device__ __forceinline__ f32x2 where_column(u32 base, u32 lane, u32 cols, u32 i, float v) {
    if (VEC) return both_2(base + lane * 8 < cols ? v : 0.f);              // all eight are in or out
    return pack_2(lane_col<VEC>(base, lane, 2 * i) < cols ? v : 0.f, lane_col<VEC>(base, lane, 2 * i + 1) < cols ? v : 0.f);
}
// One value per column, 32-bit floats or T (runtime: the branch is the same for all).
template <typename T, bool VEC>
__device__ __forceinline__ void load_vector(const ColumnVector& w, u32 base, u32 lane, u32 cols, float absent, Eight& v) {
    if (!w.p) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = both_2(absent);
    } else if (sizeof(T) != 4 && w.dtype == DT_F32) {
        load_cols<float, VEC, false>(static_cast<const float*>(w.p), base, lane, cols, v);
    } else {
        load_cols<T, VEC, false>(static_cast<const T*>(w.p), base, lane, cols, v);
    }
}

// ---- blocks of 32 values in 8 bits ------------------------------------------------------------------------------------------
// The scale of a block from its largest magnitude A (as bits): fl(A / 127) rounded up to 8 significant bits, at least 2^-126; NaN where the
// block holds one or an infinity.  It has the bits of a bfloat16.
// That is the smallest number s of 8 bits with 127 s >= A: the product is exact in fp32, and where A is above it by one unit in its last
// place, A / 127 is above s by more than half of one of its own (127 s has 1.984 or 0.992 times the significand of s), so the quotient
// does not round down to s.  A times a little less than 1 / 127 gives s or the number before it.
__device__ __forceinline__ float a8_scale(u32 largest) {
    if (largest >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const float a = __uint_as_float(largest);
    const u32 b = max((__float_as_uint(a * 0.0078740126f) + 0xffffu) & 0xffff0000u, 0x00800000u);
    return __uint_as_float(127.f * __uint_as_float(b) < a ? b + 0x10000u : b);
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
// (The products one by one: a product and a sum of two lanes each become one fused instruction, whatever their rounding says, and a
// code depends on the product's own rounding.)
__device__ __forceinline__ f32x2 a8_steps(f32x2 v, float inverse) {
    return add_2(pack_2(__fmul_rn(low_2(v), inverse), __fmul_rn(high_2(v), inverse)), both_2(12582912.f));
}
__device__ __forceinline__ u32 a8_codes(f32x2 ab, f32x2 cd, float inverse) {
    const f32x2 p = a8_steps(ab, inverse), q = a8_steps(cd, inverse);
    return __byte_perm(__byte_perm((u32)p, (u32)(p >> 32), 0x0040), __byte_perm((u32)q, (u32)(q >> 32), 0x0040), 0x5410);
}
// Bytes i and j of words of codes that were turned to 0 .. 255 (^ 0x80808080), times their scales.
__device__ __forceinline__ f32x2 a8_values(u32 turned_a, u32 i, u32 turned_b, u32 j, f32x2 scale) {
    const u32 a = __byte_perm(turned_a, 0x4b000000u, 0x7440u + i), b = __byte_perm(turned_b, 0x4b000000u, 0x7440u + j);
    return mul_2(add_2((u64)a | (u64)b << 32, both_2(-8388736.f)), scale);
}
__device__ __forceinline__ void a8_eight(u32 first, u32 second, float scale, Eight& v) {
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        const u32 w = (i < 2 ? first : second) ^ 0x80808080u;
        v[i] = a8_values(w, (2 * i) % 4, w, (2 * i + 1) % 4, both_2(scale));
    }
}
// The larger magnitude; NaN if one is.
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
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
__device__ __forceinline__ void store_kept(const Kept& k, u64 row, u32 base, u32 lane, const Eight& v) {
    unsigned char* codes = k.codes + row * k.blocks * A8_BLOCK;
    unsigned short* scales = k.scales + row * k.blocks;
    if constexpr (VEC) {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = larger(larger(m, low_2(v[i])), high_2(v[i]));
        u32 top = __float_as_uint(m) & 0x7fffffffu;
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float s = a8_scale(top);
        const float inverse = a8_inverse(s);
        uint2 q = make_uint2(a8_codes(v[0], v[1], inverse), a8_codes(v[2], v[3], inverse));
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
            const float x = e % 2 ? high_2(v[e / 2]) : low_2(v[e / 2]);
            const u32 top = __reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu);
            const float s = a8_scale(top);
            const u32 q = top >= 0x7f800000u ? 0u : a8_codes(x, 0.f, 0.f, 0.f, a8_inverse(s));
            codes[b * A8_BLOCK + lane] = (unsigned char)q;
            if (lane == 0) scales[b] = (unsigned short)(__float_as_uint(s) >> 16);
        }
    }
}

template <bool VEC>
struct RawKept {                                   // a lane's eight codes and their scales as they lie in memory
    u32 q[VEC ? 2 : 8];
    unsigned short s[VEC ? 1 : 8];
    // codes, scales: of the row
    __device__ __forceinline__ void load(const unsigned char* codes, const unsigned short* scales, u32 blocks, u32 base, u32 lane) {
        if constexpr (VEC) {
            const u32 c = base + lane * 8;
            const bool there = c / A8_BLOCK < blocks;
            const uint2 w = there ? __ldg(reinterpret_cast<const uint2*>(codes + c)) : make_uint2(0u, 0u);
            q[0] = w.x;
            q[1] = w.y;
            s[0] = there ? __ldg(scales + c / A8_BLOCK) : 0;
        } else {
#pragma unroll
            for (u32 e = 0; e < 8; ++e) {
                const u32 b = base / A8_BLOCK + e;
                q[e] = b < blocks ? codes[b * A8_BLOCK + lane] : 0u;
                s[e] = b < blocks ? scales[b] : 0;
            }
        }
    }
    __device__ __forceinline__ void load(const Kept& k, u64 row, u32 base, u32 lane) {
        load(k.codes + row * k.blocks * A8_BLOCK, k.scales + row * k.blocks, k.blocks, base, lane);
    }
    __device__ __forceinline__ void values(Eight& v) const {
        if constexpr (VEC) {
            a8_eight(q[0], q[1], __uint_as_float((u32)s[0] << 16), v);
        } else {
#pragma unroll
            for (u32 i = 0; i < 4; ++i)
                v[i] = a8_values(q[2 * i] ^ 0x80u, 0, q[2 * i + 1] ^ 0x80u, 0, (u64)((u32)s[2 * i] << 16) | (u64)((u32)s[2 * i + 1] << 16) << 32);
        }
    }
};
#endif

}  // namespace excp
