// Microscaled 4-bit matrices: tensor scale, quantisation, and back.
//
// A block of B consecutive values of a row shares a scale; a value is held as the nearest of
// 0, .5, 1, 1.5, 2, 3, 4, 6 (and sign) to value / scale.  Definitions, byte for byte: include/excp.h.
//
// Work split: a warp takes 256 columns (one tile) of the four rows l, l + 32, l + 64, l + 96 of a row tile, two rows at a
// time: a half-warp has a row, a lane 16 consecutive values of it, so that
//   - a lane's values are one or two 32-byte loads, all four rows in flight,
//   - a block's largest magnitude is in the lane (blocks of 16) or one shuffle away, and its scale is worked out once or twice,
//   - a row's codes leave as 128 consecutive bytes, and its scales as words of the layout the tensor core reads
//     (row 32 c + l of piece j at byte 16 l + 4 c).
// Rows that do not start on 32 bytes go through shared memory: loaded and stored value by value, neighbouring lanes
// neighbouring values.
// Bound and time: 32000 x 4096 fp32 85 us, back 90 us (HBM, 7.0 and 6.6 TB/s of what must move); 11008 x 4096 bf16, blocks of
// 16: 24 us (issue), back 19.6 us (HBM, 5.9 TB/s), tensor scale 12.5 us (L2 and HBM).
#include <type_traits>

#include "mx4_codes.cuh"
#include "score_launch.cuh"

namespace excp {
namespace {

constexpr int WARPS = 8;

// How a matrix in ordinary layout is reached: its rows all start on 32 bytes, on 16, or anywhere.
enum Reach { REACH_32, REACH_16, REACH_ANY };

// Values c0 .. c0 + 15 of a row of `cols`, 0 past the end; p: the first one.
__device__ __forceinline__ void load32(const void* p, uint4& a, uint4& b) {
    asm volatile("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
template <typename T> struct Sixteen { uint4 w[sizeof(T)]; };          // 16 values as words
template <typename T, int REACH>
__device__ __forceinline__ void load_words(const T* p, u64 left, Sixteen<T>& v) {      // left: values of the row from p on
    if (left >= 16) {
        const uint4* q = reinterpret_cast<const uint4*>(p);
#pragma unroll
        for (u32 i = 0; i < sizeof(T); i += 2) {
            if (REACH == REACH_32) load32(q + i, v.w[i], v.w[i + 1]);
            else { v.w[i] = __ldg(q + i); v.w[i + 1] = __ldg(q + i + 1); }
        }
        return;
    }
    T* h = reinterpret_cast<T*>(&v);
#pragma unroll
    for (u32 k = 0; k < 16; ++k) wput(h, k, k < left ? wget(p, k) : 0.f);
}
template <typename T, int REACH>
__device__ __forceinline__ void store_words(T* p, u64 left, const Sixteen<T>& v) {
    if (left >= 16) {
        uint4* q = reinterpret_cast<uint4*>(p);
#pragma unroll
        for (u32 i = 0; i < sizeof(T); i += 2) {
            if (REACH == REACH_32) store32(q + i, v.w[i], v.w[i + 1]);
            else { q[i] = v.w[i]; q[i + 1] = v.w[i + 1]; }
        }
        return;
    }
    const T* h = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (u32 k = 0; k < 16; ++k) if (k < left) p[k] = h[k];
}

// Values from the 16-byte boundary at or before p to p.
template <typename T> __device__ __forceinline__ u32 offset16(const T* p) { return (u32)(reinterpret_cast<uintptr_t>(p) & 15) / (u32)sizeof(T); }

// Pattern of the largest magnitude of 16 values (at or above NONFINITE_BITS where there is an infinity or a NaN).
__device__ __forceinline__ u32 largest_bits(const Sixteen<float>& v) {
    const u32* b = reinterpret_cast<const u32*>(&v);
    u32 m = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, b[k] & 0x7fffffffu);
    return m;
}
template <typename T>
__device__ __forceinline__ u32 largest_bits(const Sixteen<T>& v) {
    typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type T2;
    const T2* h = reinterpret_cast<const T2*>(&v);
    T2 m = __habs2(h[0]);
#pragma unroll
    for (int k = 1; k < 8; ++k) m = __hmax2_nan(m, __habs2(h[k]));
    const T* e = reinterpret_cast<const T*>(&m);
    return max(__float_as_uint(wget(e, 0)) & 0x7fffffffu, __float_as_uint(wget(e, 1)) & 0x7fffffffu);
}

// ---- tensor scale: max |x| / 2688, rounded up to 8 significant bits -----------------
// A warp takes 512 values of a row at a time, counted from the row's first 32-byte boundary; the warp of a row's first
// values also takes what lies before it.
template <typename T>
__global__ void __launch_bounds__(256) tensor_scale_kernel(const T* __restrict__ x, u64 rows, u64 cols, u64 stride, u32 chunks,
                                                           u32* words, float* scale_out) {
    wait_for_previous();
    let_next_start();
    u32 best = 0;
    auto take = [&](u32 m) {
        if (m < NONFINITE_BITS && m > best) best = m;
    };
    const u32 lane = threadIdx.x & 31;
    const u64 total = rows * chunks, step = (u64)gridDim.x * 8;
    for (u64 i = (u64)blockIdx.x * 8 + (threadIdx.x >> 5); i < total; i += step) {
        const u64 r = i / chunks, chunk = i - r * chunks;
        const T* const row = x + r * stride;
        const u64 head = min((u64)((32 - (reinterpret_cast<uintptr_t>(row) & 31)) & 31) / sizeof(T), cols);
        if (chunk == 0 && lane < head) take(__float_as_uint(wget(row, lane)) & 0x7fffffffu);
        const u64 c0 = head + chunk * 512;
        if (c0 >= cols) continue;
        const T* p = row + c0;
        const u64 left = cols - c0;
        if (left < 512) {
#pragma unroll
            for (u32 k = 0; k < 16; ++k) if (lane + 32 * k < left) take(__float_as_uint(wget(p, lane + 32 * k)) & 0x7fffffffu);
        } else {
            Sixteen<T> v;
            load_words<T, REACH_32>(p + lane * 16, 16, v);
            const u32 m = largest_bits(v);
            if (m < NONFINITE_BITS) {
                take(m);
            } else {                               // the finite ones one by one
                const T* h = reinterpret_cast<const T*>(&v);
#pragma unroll
                for (u32 k = 0; k < 16; ++k) take(__float_as_uint(wget(h, k)) & 0x7fffffffu);
            }
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    __shared__ u32 part[8];
    if (lane == 0) part[threadIdx.x >> 5] = best;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 8; ++w) best = max(best, part[w]);
    atomicMax(&words[0], best);
    __threadfence();
    if (atomicAdd(&words[1], 1u) != gridDim.x - 1) return;
    __threadfence();                               // the last block: every maximum is in
    best = atomicExch(&words[0], 0u);
    words[1] = 0;
    const float q = __fdiv_rn(__uint_as_float(best), 2688.f);
    // 8 significant bits: the upper half of the pattern, or of a subnormal's the 8 from its leading one on; a carry is right as it is
    const u32 bits = __float_as_uint(q);
    const u32 low = (1u << (bits >= 0x00800000u ? 16 : max(24 - __clz(bits), 0))) - 1u;
    scale_out[0] = q > 0.f ? __uint_as_float((bits + low) & ~low) : 1.f;
}

// Where a warp works: tile (rt, ct), rows l + 32 c.  A tile is four blocks of eight warps.  (Four values of l to a warp, and
// the addresses worked out once for them, were slower: 11008 x 4096 bf16 30 us against 26, too few warps.)
struct Place {
    u32 ct, l, height;
    u64 offset, row0;
    __device__ __forceinline__ Place(u64 rows, u32 col_tiles, int fmt) {
        const u32 tile = blockIdx.x >> 2, rt = tile / col_tiles;
        l = (blockIdx.x & 3) * WARPS + (threadIdx.x >> 5);
        ct = tile - rt * col_tiles;
        height = mx4_tile_height(rows, rt);
        offset = mx4_tile_offset(rows, col_tiles, fmt, rt, ct);
        row0 = (u64)rt * MX4_ROWS + l;
    }
};

// 16 bits: 14.9 instructions per value, so as many warps as 42 registers allow (11008 x 4096 bf16, blocks of 16: 23.9 us
// with six blocks per SM, 25.9 with four).
template <typename T, int FMT, int REACH>
__global__ void __launch_bounds__(WARPS * 32, sizeof(T) == 2 ? 6 : 4) quantize_kernel(const T* __restrict__ x, u64 rows, u64 cols, u64 stride, u32 col_tiles,
                                                              const float* __restrict__ tensor_scale, unsigned char* __restrict__ out) {
    wait_for_previous();
    let_next_start();                              // a product of this matrix may set itself up and fetch the other one
    __shared__ __align__(16) T buffer[REACH == REACH_ANY ? WARPS : 1][REACH == REACH_ANY ? 4 : 1][MX4_COLS];
    const u32 warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, part = lane & 15;
    const Place at(rows, col_tiles, FMT);
    unsigned char* const dst = out + at.offset;
    const u64 first = (u64)at.ct * MX4_COLS, c0 = first + part * 16;

    Sixteen<T> v[2];
    if (REACH == REACH_ANY) {
        constexpr u32 PER = MX4_COLS / 32;
        // values one by one, everything on its way before anything is stored (whole 16-byte words, cut to the row's offset as
        // they leave the buffer, were slower: 15808 x 6009 fp16 72 us against 65; the kernel is bound by its instructions)
        T t[4][PER];
#pragma unroll
        for (u32 c = 0; c < 4; ++c) {
            const u64 row = at.row0 + 32 * c;
            const T* p = x + row * stride + first + lane;
            const u32 n = row < rows ? (u32)min(cols - first, (u64)MX4_COLS) : 0u;
#pragma unroll
            for (u32 k = 0; k < PER; ++k) t[c][k] = T(0.f);
            if (n == MX4_COLS) {
#pragma unroll
                for (u32 k = 0; k < PER; ++k) t[c][k] = __ldg(p + 32 * k);
            } else {
#pragma unroll
                for (u32 k = 0; k < PER; ++k) if (lane + 32 * k < n) t[c][k] = p[32 * k];
            }
        }
#pragma unroll
        for (u32 c = 0; c < 4; ++c)
#pragma unroll
            for (u32 k = 0; k < PER; ++k) buffer[warp][c][lane + 32 * k] = t[c][k];
        __syncwarp();
#pragma unroll
        for (u32 i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const Sixteen<T>*>(&buffer[warp][2 * i + half][part * 16]);
    } else {
#pragma unroll
        for (u32 i = 0; i < 2; ++i) {
            const u64 row = at.row0 + 32 * (2 * i + half);
            load_words<T, REACH>(x + row * stride + c0, row < rows && c0 < cols ? cols - c0 : 0, v[i]);
        }
    }
    float g = 1.f;
    if (FMT == MX4_E4M3_16 && tensor_scale) g = __ldg(tensor_scale);
    const float six_g = 6.f * g;
#pragma unroll
    for (u32 i = 0; i < 2; ++i) {
        const u32 c = 2 * i + half, r = at.l + 32 * c;
        u32 m = largest_bits(v[i]);
        if (FMT == MX4_E8M0_32) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        float f[16];
        const T* h = reinterpret_cast<const T*>(&v[i]);
#pragma unroll
        for (u32 k = 0; k < 16; ++k) f[k] = wget(h, k);
        u32 byte = FMT == MX4_E8M0_32 ? scale_e8m0(f, m) : scale_e4m3(f, m, g, six_g);
        // no row here, or no such block in the row: scale byte 0
        constexpr u64 B = (u64)mx4_block(FMT);
        if (at.row0 + 32 * c >= rows || c0 / B * B >= cols) byte = 0;
        // lane `part` has half a chunk of 16 bytes
        if (r < at.height)
            *reinterpret_cast<uint2*>(dst + r * 128 + (((part >> 1) ^ (r & 7)) << 4) + ((part & 1) << 3)) = make_uint2(codes_of<FMT>(f), codes_of<FMT>(f + 8));
        // the bytes of four blocks as a word
        constexpr u32 STEP = (u32)mx4_block(FMT) / 16;          // lanes to a block
        u32 word = byte | __shfl_xor_sync(0xffffffffu, byte, STEP) << 8;
        word |= __shfl_xor_sync(0xffffffffu, word, 2 * STEP) << 16;
        if (part % (4 * STEP) == 0)
            *reinterpret_cast<u32*>(dst + at.height * 128 + part / (4 * STEP) * MX4_PIECE + at.l * 16 + c * 4) = word;
    }
}

// ---- and back ------------------------------------------------------------------------------
// Eight codes as fp16 values, two to a word.
__device__ __forceinline__ void values_of(u32 codes, __half2 (&v)[4]) {
    u32 w[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const __half2*>(&w[i]);
}

template <typename T, int FMT, int REACH>
__global__ void __launch_bounds__(WARPS * 32) dequantize_kernel(const unsigned char* __restrict__ packed, u64 rows, u64 cols,
                                                                u32 col_tiles, const float* __restrict__ tensor_scale,
                                                                T* __restrict__ out, u64 stride) {
    constexpr u32 S = sizeof(T), WORDS = MX4_COLS * S / 16;      // 16-byte words to 16 values and to a row's part in the tile
    __shared__ uint4 buffer[REACH == REACH_ANY ? WARPS : 1][REACH == REACH_ANY ? 4 : 1][WORDS + 1];
    const u32 warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, part = lane & 15;
    const Place at(rows, col_tiles, FMT);
    wait_for_previous();
    let_next_start();
    if (at.row0 >= rows) return;                   // the whole warp
    const unsigned char* const src = packed + at.offset;
    const u64 first = (u64)at.ct * MX4_COLS, c0 = first + part * 16;
    constexpr u32 STEP = (u32)mx4_block(FMT) / 16;
    const u32 block = part / STEP;
    uint2 codes[2];
    u32 byte[2];
#pragma unroll
    for (u32 i = 0; i < 2; ++i) {
        const u32 c = 2 * i + half, r = at.l + 32 * c;
        const bool there = at.row0 + 32 * c < rows;
        codes[i] = there ? __ldg(reinterpret_cast<const uint2*>(src + r * 128 + (((part >> 1) ^ (r & 7)) << 4) + ((part & 1) << 3))) : make_uint2(0u, 0u);
        byte[i] = there ? __ldg(src + at.height * 128 + (block >> 2) * MX4_PIECE + at.l * 16 + c * 4 + (block & 3)) : 0u;
    }
    float g = 1.f;
    if (FMT == MX4_E4M3_16 && tensor_scale) g = __ldg(tensor_scale);
#pragma unroll
    for (u32 i = 0; i < 2; ++i) {
        const u64 row = at.row0 + 32 * (2 * i + half);
        __half2 q[8];
        values_of(codes[i].x, reinterpret_cast<__half2 (&)[4]>(q[0]));
        values_of(codes[i].y, reinterpret_cast<__half2 (&)[4]>(q[4]));
        float by;                                  // what the fp16 products below are multiplied with
        if (FMT == MX4_E4M3_16) {                  // code times scale has six significant bits and fits fp16
            const __half s = __half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte[i], __NV_E4M3));
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] = __hmul2(q[k], __half2half2(s));
            by = g;
        } else {
            by = byte[i] == 0xffu ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte[i] ? byte[i] << 23 : 0x00400000u);   // 2^(byte - 127), subnormal at 0
        }
        Sixteen<T> v;
        T* h = reinterpret_cast<T*>(&v);
        const u64 by2 = f2_pack(by, by);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 f = __half22float2(q[k]);
            float a, b;
            f2_unpack(f2_mul(f2_pack(f.x, f.y), by2), a, b);
            wput(h, 2 * k, a);
            wput(h, 2 * k + 1, b);
        }
        if (REACH == REACH_ANY) {
#pragma unroll
            for (u32 j = 0; j < S; ++j) buffer[warp][2 * i + half][part * S + j] = v.w[j];
        } else if (row < rows && c0 < cols) {
            store_words<T, REACH>(out + row * stride + c0, cols - c0, v);
        }
    }
    if (REACH == REACH_ANY) {
        __syncwarp();
        constexpr u32 N = 16 / S;
        const u32 n = (u32)min(cols - first, (u64)MX4_COLS);
        // the 16-byte words that lie wholly in a row's part
#pragma unroll
        for (u32 c = 0; c < 4; ++c) {
            const u64 row = at.row0 + 32 * c;
            T* p = out + row * stride + first;
            const u32 head = (N - offset16(p)) % N;
            const uint4* w = &buffer[warp][c][0];
#pragma unroll
            for (u32 k = 0; k < WORDS / 32; ++k) {
                const u32 word = lane + 32 * k;
                if (row < rows && head + (word + 1) * N <= n) __stcs(reinterpret_cast<uint4*>(p + head) + word, cut16(w[word], w[word + 1], head * S));
            }
        }
        // and the values before and after them: 2 x N lanes to a row
#pragma unroll
        for (u32 k = 0; k < 4 * 2 * N / 32; ++k) {
            const u32 i = lane + 32 * k, c = i / (2 * N), at_edge = i % N;
            const u64 row = at.row0 + 32 * c;
            T* p = out + row * stride + first;
            const u32 head = min((N - offset16(p)) % N, n), whole = (n - head) / N * N;
            const u32 value = i / N % 2 ? head + whole + at_edge : at_edge;
            if (row < rows && (i / N % 2 ? value < n : value < head)) p[value] = reinterpret_cast<const T*>(&buffer[warp][c][0])[value];
        }
    }
}

template <typename T>
int reach(const void* p, u64 rows, u64 stride) {
    const u64 bits = reinterpret_cast<uintptr_t>(p) | (rows <= 1 ? 0 : stride * sizeof(T));
    return (bits & 31) == 0 ? REACH_32 : (bits & 15) == 0 ? REACH_16 : REACH_ANY;
}
#define EXCP_REACH(r, CALL) ((r) == REACH_32 ? CALL(REACH_32) : (r) == REACH_16 ? CALL(REACH_16) : CALL(REACH_ANY))

template <typename T>
void tensor_scale_as(int sms, cudaStream_t s, const RowsIn& x, u32* words, float* out) {
    const u32 chunks = (u32)((x.cols + 511) / 512);
    const u64 want = (x.rows * chunks + 7) / 8;
    const u32 grid = (u32)(want < 1 ? 1 : (want > (u64)sms * 8 ? (u64)sms * 8 : want));
    launch_chained(tensor_scale_kernel<T>, grid, 256, 0, 0, s, static_cast<const T*>(x.p), x.rows, x.cols, x.stride, chunks, words, out);
}
template <typename T, int FMT, int REACH>
void quantize_as(cudaStream_t s, const RowsIn& x, const float* tensor_scale, unsigned char* out) {
    const u32 ct = mx4_col_tiles(x.cols);
    launch_chained(quantize_kernel<T, FMT, REACH>, mx4_row_tiles(x.rows) * ct * 4, WARPS * 32, 0, 0, s, static_cast<const T*>(x.p), x.rows, x.cols,
                   x.stride, ct, tensor_scale, out);
}
template <typename T, int FMT, int REACH>
void dequantize_as(cudaStream_t s, const unsigned char* packed, u64 rows, u64 cols, const float* tensor_scale, void* out, u64 stride) {
    const u32 ct = mx4_col_tiles(cols);
    launch_chained(dequantize_kernel<T, FMT, REACH>, mx4_row_tiles(rows) * ct * 4, WARPS * 32, 0, 0, s, packed, rows, cols, ct, tensor_scale,
                   static_cast<T*>(out), stride);
}

}  // namespace

void launch_mx4_tensor_scale(int sms, cudaStream_t s, const RowsIn& x, u32* words, float* scale_out) {
    if (x.dtype == DT_F32) tensor_scale_as<float>(sms, s, x, words, scale_out);
    else if (x.dtype == DT_F16) tensor_scale_as<__half>(sms, s, x, words, scale_out);
    else tensor_scale_as<__nv_bfloat16>(sms, s, x, words, scale_out);
}

void launch_mx4_quantize(int, cudaStream_t s, const RowsIn& x, int fmt, const float* tensor_scale, unsigned char* out) {
#define EXCP_Q4(R) quantize_as<T, MX4_E4M3_16, R>(s, x, tensor_scale, out)
#define EXCP_Q8(R) quantize_as<T, MX4_E8M0_32, R>(s, x, tensor_scale, out)
    auto run = [&](auto zero) {
        typedef decltype(zero) T;
        const int r = reach<T>(x.p, x.rows, x.stride);
        if (fmt == MX4_E4M3_16) EXCP_REACH(r, EXCP_Q4);
        else EXCP_REACH(r, EXCP_Q8);
    };
    if (x.dtype == DT_F32) run(float());
    else if (x.dtype == DT_F16) run(__half());
    else run(__nv_bfloat16());
#undef EXCP_Q4
#undef EXCP_Q8
}

void launch_mx4_dequantize(int, cudaStream_t s, const unsigned char* packed, u64 rows, u64 cols, int fmt,
                           const float* tensor_scale, void* out, int dtype, u64 stride) {
#define EXCP_D4(R) dequantize_as<T, MX4_E4M3_16, R>(s, packed, rows, cols, tensor_scale, out, stride)
#define EXCP_D8(R) dequantize_as<T, MX4_E8M0_32, R>(s, packed, rows, cols, tensor_scale, out, stride)
    auto run = [&](auto zero) {
        typedef decltype(zero) T;
        const int r = reach<T>(out, rows, stride);
        if (fmt == MX4_E4M3_16) EXCP_REACH(r, EXCP_D4);
        else EXCP_REACH(r, EXCP_D8);
    };
    if (dtype == DT_F32) run(float());
    else if (dtype == DT_F16) run(__half());
    else run(__nv_bfloat16());
#undef EXCP_D4
#undef EXCP_D8
}

}  // namespace excp
