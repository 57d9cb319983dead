// Log probabilities of given tokens, entropy and the likeliest alternatives of rows of logits, and the
// gradient of the first two.
//
//   z = scale * logits, m = max z, d = z - m, S = sum exp d, T = sum d exp d
//   log p_v = d_v - log S,   entropy = log S - T / S
//   gradient: scale * (g_lp ([v = token] - p_v) - g_h p_v (log p_v + entropy))
//
// One pass keeps (m, S, T) per thread and rescales when the maximum moves: with delta = m - m' the sums become
// S e^delta and (T + S delta) e^delta.  Everything is fp32; subtracting the maximum before the sums keeps their
// relative error at a few roundings.  A forbidden word (logit -inf) adds 0 to both sums.
#include "score.cuh"

namespace excp {
namespace {

constexpr int BLOCK = 256;
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float LOG2E = 1.4426950408889634f;
constexpr float FAR = -150.f;                      // exp of less is 0 in fp32

// d below FAR counts as FAR: exp is 0 there and d exp d stays a number.  NaN stays NaN.
__device__ __forceinline__ float near_part(float d) { return d < FAR ? FAR : d; }

struct Sums {
    float m, s, t;
};
__device__ __forceinline__ void add_value(Sums& a, float z) {
    if (z > a.m) {
        const float f = near_part(a.m - z);
        const float e = exp2f(f * LOG2E);
        a.t = a.s > 0.f ? (a.t + a.s * f) * e : 0.f;
        a.s *= e;
        a.m = z;
    }
    if (z == NEG_INF) return;
    const float d = near_part(z - a.m);
    const float e = exp2f(d * LOG2E);
    a.s += e;
    a.t = fmaf(d, e, a.t);
}
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
    Sums r;
    r.m = fmaxf(a.m, b.m);
    if (r.m == NEG_INF) { r.s = a.s + b.s; r.t = a.t + b.t; return r; }
    const float fa = near_part(a.m - r.m), fb = near_part(b.m - r.m);
    const float ea = exp2f(fa * LOG2E), eb = exp2f(fb * LOG2E);
    r.s = a.s * ea + b.s * eb;
    r.t = (a.t + a.s * fa) * ea + (b.t + b.s * fb) * eb;
    return r;
}

// Order of the alternatives: larger logit first, of equal ones the lower index; -0 counts as 0, NaN as largest.
__device__ __forceinline__ u64 order_key(float v, u32 index) {
    u32 b = __float_as_uint(v + 0.f);
    if (v != v) b = 0x7fffffffu;
    b = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return ((u64)b << 32) | (0xffffffffu - index);
}

template <typename T>
__global__ void __launch_bounds__(BLOCK) logprobs_kernel(const T* __restrict__ logits, u32 vocab, u64 stride,
                                                         const long long* __restrict__ tokens, float scale, LogprobsOut out) {
    const u64 row = blockIdx.x;
    const T* x = logits + row * stride;
    Sums a{NEG_INF, 0.f, 0.f};
    for (u32 i = threadIdx.x; i < vocab; i += BLOCK) add_value(a, wget(x, i) * scale);
    __shared__ Sums part[BLOCK / 32];
    __shared__ u64 best[BLOCK / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const Sums b{__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.t, o)};
        a = join(a, b);
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
    __syncthreads();
    a = part[0];
    for (int w = 1; w < BLOCK / 32; ++w) a = join(a, part[w]);
    const float log_s = logf(a.s);
    const bool empty = a.m == NEG_INF && a.s == 0.f;
    auto log_p = [&](float v) { return empty ? NEG_INF : v * scale - a.m - log_s; };
    if (threadIdx.x == 0) {
        const long long t = tokens[row];
        const float h = empty ? 0.f : log_s - a.t / a.s;
        out.logprob[row] = t < 0 ? 0.f : t < (long long)vocab ? log_p(wget(x, (u64)t)) : __uint_as_float(0x7fffffffu);
        if (out.entropy) out.entropy[row] = h;
        if (out.row_stats) reinterpret_cast<float4*>(out.row_stats)[row] = make_float4(a.m, a.s, h, 0.f);
    }
    u64 last = ~0ull;
    for (int k = 0; k < out.top; ++k) {
        u64 mine = 0;
        for (u32 i = threadIdx.x; i < vocab; i += BLOCK) {
            const u64 key = order_key(wget(x, i), i);
            if (key < last && key > mine) mine = key;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const u64 other = __shfl_xor_sync(0xffffffffu, mine, o);
            if (other > mine) mine = other;
        }
        if ((threadIdx.x & 31) == 0) best[threadIdx.x >> 5] = mine;
        __syncthreads();
        for (int w = 0; w < BLOCK / 32; ++w) if (best[w] > mine) mine = best[w];
        __syncthreads();
        if (threadIdx.x == 0) {
            const u32 index = 0xffffffffu - (u32)mine;
            out.top_index[row * out.top + k] = index;
            out.top_logprob[row * out.top + k] = log_p(wget(x, index));
        }
        last = mine;
    }
}

template <typename T>
__global__ void __launch_bounds__(BLOCK) grad_kernel(const T* logits, u32 vocab, u64 stride, const long long* __restrict__ tokens,
                                                     float scale, const float* __restrict__ row_stats, const float* __restrict__ g_logprob,
                                                     const float* __restrict__ g_entropy, T* grad, u64 grad_stride) {
    const u64 row = blockIdx.x;
    const float4 st = __ldg(reinterpret_cast<const float4*>(row_stats) + row);
    const long long t = tokens[row];
    float gl = g_logprob && t >= 0 ? __ldg(g_logprob + row) : 0.f;
    if (t >= (long long)vocab) gl = __uint_as_float(0x7fffffffu);
    const float gh = g_entropy ? __ldg(g_entropy + row) : 0.f;
    const bool empty = st.x == NEG_INF && st.y == 0.f;
    const float log_s = logf(st.y), inv_s = 1.f / st.y;
    const T* x = logits + row * stride;
    T* y = grad + row * grad_stride;
    for (u32 i = threadIdx.x; i < vocab; i += BLOCK) {
        const float d = near_part(wget(x, i) * scale - st.x);
        const float p = exp2f(d * LOG2E) * inv_s;
        const float one = (long long)i == t ? 1.f : 0.f;
        const float v = scale * (gl * (one - p) - gh * p * (d - log_s + st.z));
        wput(y, i, empty ? 0.f : v);
    }
}

}  // namespace

void launch_token_logprobs(int, cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const LogprobsOut& out) {
#define EXCP_L(T) logprobs_kernel<T><<<(u32)x.rows, BLOCK, 0, s>>>(static_cast<const T*>(x.p), (u32)x.cols, x.stride, tokens, scale, out)
    if (x.dtype == DT_F32) EXCP_L(float);
    else if (x.dtype == DT_F16) EXCP_L(__half);
    else EXCP_L(__nv_bfloat16);
#undef EXCP_L
}

void launch_token_logprobs_grad(int, cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const float* row_stats,
                                const float* g_logprob, const float* g_entropy, void* grad, u64 grad_stride) {
#define EXCP_G(T) grad_kernel<T><<<(u32)x.rows, BLOCK, 0, s>>>(static_cast<const T*>(x.p), (u32)x.cols, x.stride, tokens, scale, row_stats, \
                                                              g_logprob, g_entropy, static_cast<T*>(grad), grad_stride)
    if (x.dtype == DT_F32) EXCP_G(float);
    else if (x.dtype == DT_F16) EXCP_G(__half);
    else EXCP_G(__nv_bfloat16);
#undef EXCP_G
}

}  // namespace excp
