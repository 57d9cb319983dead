// Microscaled 4-bit matrices: tensor scale, quantisation, and back.
//
// A block of B consecutive values of a row shares a scale; a value is held as the nearest of
// 0, .5, 1, 1.5, 2, 3, 4, 6 (and sign) to value / scale.  Definitions, byte for byte: include/excp.h.
//
// Work split: a warp takes 256 columns (one tile) of the four rows l, l + 32, l + 64, l + 96 of a row tile;
// lane i holds the eight consecutive values 8 i .. 8 i + 7 of each, so that
//   - a load of the warp is 512 (16-bit) or 1024 (fp32) consecutive bytes of a row, four rows in flight,
//   - a block's largest magnitude is two shuffles (B = 32) or one (B = 16) away,
//   - a row's codes leave as 128 consecutive bytes, and the four rows' scales of a block of columns as whole
//     16-byte groups of the layout the tensor core reads (row 32 c + l of piece j at byte 16 l + 4 c).
#include "mx4_codes.cuh"
#include "mx4_pipe.cuh"

namespace excp {
namespace {

constexpr int WARPS = 8;

// ---- tensor scale: max |x| / 2688, rounded up to 8 significant bits -----------------
template <typename T>
__global__ void __launch_bounds__(256) tensor_scale_kernel(const T* __restrict__ x, u64 rows, u64 cols, u64 stride, bool vec,
                                                           u32* words, float* scale_out) {
    u32 best = 0;
    auto take = [&](float v) {
        const u32 m = __float_as_uint(v) & 0x7fffffffu;
        if (m < NONFINITE_BITS && m > best) best = m;
    };
    const u64 groups = (cols + 7) / 8;
    const u64 total = rows * groups;
    for (u64 i = (u64)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (u64)gridDim.x * blockDim.x) {
        const u64 r = i / groups, c = (i - r * groups) * 8;
        const T* p = x + r * stride + c;
        float v[8];
        if (vec && c + 8 <= cols) {
            load8(p, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) take(v[k]);
        } else {
            for (int k = 0; k < 8 && c + k < cols; ++k) take(wget(p, k));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    __shared__ u32 part[8];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = best;
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
    // 8 significant bits = the upper half of the pattern; q > 0 keeps at least one
    scale_out[0] = q > 0.f ? __uint_as_float((__float_as_uint(q) + 0xffffu) & 0xffff0000u) : 1.f;
}

template <typename T, int FMT>
__global__ void __launch_bounds__(WARPS * 32) quantize_kernel(const T* __restrict__ x, u64 rows, u64 cols, u64 stride, bool vec,
                                                              u32 col_tiles, u64 tasks, const float* __restrict__ tensor_scale,
                                                              unsigned char* __restrict__ out) {
    let_next_start();                              // a product of this matrix may set itself up and fetch the other one
    const u64 task = (u64)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const u32 lane = threadIdx.x & 31;
    const u32 l = (u32)(task & 31);
    const u64 tile = task >> 5;
    const u32 rt = (u32)(tile / col_tiles), ct = (u32)(tile - (u64)rt * col_tiles);
    const u32 height = mx4_tile_height(rows, rt);
    unsigned char* const dst = out + mx4_tile_offset(rows, col_tiles, FMT, rt, ct);
    const u64 row0 = (u64)rt * MX4_ROWS + l, c0 = (u64)ct * MX4_COLS + lane * 8;

    float g = 1.f;
    if (FMT == MX4_E4M3_16 && tensor_scale) g = __ldg(tensor_scale);
    const float six_g = 6.f * g;

    float v[4][8];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const T* p = x + (row0 + 32 * c) * stride + c0;
        if (row0 + 32 * c < rows && vec && c0 + 8 <= cols) {
            load8(p, v[c]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[c][k] = row0 + 32 * c < rows && c0 + k < cols ? wget(p, k) : 0.f;
        }
    }
    u32 bytes[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32 m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(v[c][k]) & 0x7fffffffu);
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        if (FMT == MX4_E8M0_32) m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        bytes[c] = FMT == MX4_E8M0_32 ? scale_e8m0(v[c], m) : scale_e4m3(v[c], m, g, six_g);
        // no row here, or no such block in the row: scale byte 0
        constexpr u32 B = (u32)mx4_block(FMT);
        if (row0 + 32 * c >= rows || c0 / B * B >= cols) bytes[c] = 0;
        const u32 r = l + 32 * c;
        if (r < height) *reinterpret_cast<u32*>(dst + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + ((lane & 3) << 2)) = e2m1x8(v[c]);
    }
    // scale word of row c, piece j: the bytes of blocks 4 j .. 4 j + 3, held by lanes PER apart
    constexpr int PER = mx4_block(FMT) / 8;
    const u32 piece = lane >> 2, src = min(piece, (u32)mx4_pieces(FMT) - 1) * 4 * PER;
    u32 word = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const u32 w = scale_word<FMT>(bytes[c], src);
        if ((lane & 3) == (u32)c) word = w;
    }
    if (piece < (u32)mx4_pieces(FMT))
        *reinterpret_cast<u32*>(dst + height * 128 + piece * MX4_PIECE + l * 16 + (lane & 3) * 4) = word;
}

// ---- and back ------------------------------------------------------------------------------
__device__ __forceinline__ float e2m1_value(u32 code) {
    // as fp16 bits the exponent and mantissa of a 4-bit float read 2^-14 times too small, its subnormal included
    return __half2float(__ushort_as_half((unsigned short)(((code & 7u) << 9) | ((code & 8u) << 12)))) * 16384.f;
}
template <int FMT>
__device__ __forceinline__ float scale_value(u32 byte) {
    if (FMT == MX4_E4M3_16) return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
    if (byte == 0xffu) return __uint_as_float(0x7fffffffu);
    return __uint_as_float(byte ? byte << 23 : 0x00400000u);           // 2^(byte - 127), subnormal at 0
}

template <typename T, int FMT>
__global__ void __launch_bounds__(WARPS * 32) dequantize_kernel(const unsigned char* __restrict__ packed, u64 rows, u64 cols,
                                                                u32 col_tiles, u64 tasks, const float* __restrict__ tensor_scale,
                                                                T* __restrict__ out, u64 stride, bool vec) {
    const u64 task = (u64)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const u32 lane = threadIdx.x & 31;
    const u32 l = (u32)(task & 31);
    const u64 tile = task >> 5;
    const u32 rt = (u32)(tile / col_tiles), ct = (u32)(tile - (u64)rt * col_tiles);
    const u32 height = mx4_tile_height(rows, rt);
    const unsigned char* const src = packed + mx4_tile_offset(rows, col_tiles, FMT, rt, ct);
    const u64 row0 = (u64)rt * MX4_ROWS + l, c0 = (u64)ct * MX4_COLS + lane * 8;
    float g = 1.f;
    if (FMT == MX4_E4M3_16 && tensor_scale) g = __ldg(tensor_scale);
    constexpr int PER = mx4_block(FMT) / 8;
    const u32 block = lane / PER;
    u32 word[4], byte[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const u32 r = l + 32 * c;
        const bool there = row0 + 32 * c < rows;
        word[c] = there ? *reinterpret_cast<const u32*>(src + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + ((lane & 3) << 2)) : 0u;
        byte[c] = there ? src[height * 128 + (block >> 2) * MX4_PIECE + l * 16 + c * 4 + (block & 3)] : 0u;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if (row0 + 32 * c >= rows) break;
        const float s = scale_value<FMT>(byte[c]);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[k] = e2m1_value(word[c] >> (4 * k) & 15u) * s;
            if (FMT == MX4_E4M3_16) v[k] *= g;
        }
        T* p = out + (row0 + 32 * c) * stride + c0;
        if (vec && c0 + 8 <= cols) {
            store8(p, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) if (c0 + k < cols) wput(p, k, v[k]);
        }
    }
}

// Rows that all start on 16 bytes.
template <typename T>
bool rows_aligned(const void* p, u64 rows, u64 stride) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || (stride * sizeof(T)) % 16 == 0);
}

template <typename T>
void tensor_scale_as(int sms, cudaStream_t s, const RowsIn& x, u32* words, float* out) {
    const u64 groups = x.rows * ((x.cols + 7) / 8);
    const u64 want = (groups + 255) / 256;
    const u32 grid = (u32)(want < 1 ? 1 : (want > (u64)sms * 8 ? (u64)sms * 8 : want));
    tensor_scale_kernel<T><<<grid, 256, 0, s>>>(static_cast<const T*>(x.p), x.rows, x.cols, x.stride,
                                                rows_aligned<T>(x.p, x.rows, x.stride), words, out);
}

template <typename T, int FMT>
void quantize_as(cudaStream_t s, const RowsIn& x, const float* tensor_scale, unsigned char* out) {
    const u32 ct = mx4_col_tiles(x.cols);
    const u64 tasks = (u64)mx4_row_tiles(x.rows) * ct * 32;
    quantize_kernel<T, FMT><<<(u32)((tasks + WARPS - 1) / WARPS), WARPS * 32, 0, s>>>(
        static_cast<const T*>(x.p), x.rows, x.cols, x.stride, rows_aligned<T>(x.p, x.rows, x.stride), ct, tasks, tensor_scale, out);
}
template <typename T, int FMT>
void dequantize_as(cudaStream_t s, const unsigned char* packed, u64 rows, u64 cols, const float* tensor_scale, void* out, u64 stride) {
    const u32 ct = mx4_col_tiles(cols);
    const u64 tasks = (u64)mx4_row_tiles(rows) * ct * 32;
    dequantize_kernel<T, FMT><<<(u32)((tasks + WARPS - 1) / WARPS), WARPS * 32, 0, s>>>(
        packed, rows, cols, ct, tasks, tensor_scale, static_cast<T*>(out), stride, rows_aligned<T>(out, rows, stride));
}

}  // namespace

void launch_mx4_tensor_scale(int sms, cudaStream_t s, const RowsIn& x, u32* words, float* scale_out) {
    if (x.dtype == DT_F32) tensor_scale_as<float>(sms, s, x, words, scale_out);
    else if (x.dtype == DT_F16) tensor_scale_as<__half>(sms, s, x, words, scale_out);
    else tensor_scale_as<__nv_bfloat16>(sms, s, x, words, scale_out);
}

void launch_mx4_quantize(int, cudaStream_t s, const RowsIn& x, int fmt, const float* tensor_scale, unsigned char* out) {
#define EXCP_Q(T) (fmt == MX4_E4M3_16 ? quantize_as<T, MX4_E4M3_16>(s, x, tensor_scale, out) : quantize_as<T, MX4_E8M0_32>(s, x, tensor_scale, out))
    if (x.dtype == DT_F32) EXCP_Q(float);
    else if (x.dtype == DT_F16) EXCP_Q(__half);
    else EXCP_Q(__nv_bfloat16);
#undef EXCP_Q
}

void launch_mx4_dequantize(int, cudaStream_t s, const unsigned char* packed, u64 rows, u64 cols, int fmt,
                           const float* tensor_scale, void* out, int dtype, u64 stride) {
#define EXCP_D(T) (fmt == MX4_E4M3_16 ? dequantize_as<T, MX4_E4M3_16>(s, packed, rows, cols, tensor_scale, out, stride) \
                                      : dequantize_as<T, MX4_E8M0_32>(s, packed, rows, cols, tensor_scale, out, stride))
    if (dtype == DT_F32) EXCP_D(float);
    else if (dtype == DT_F16) EXCP_D(__half);
    else EXCP_D(__nv_bfloat16);
#undef EXCP_D
}

}  // namespace excp
