// Log probabilities of given tokens, entropy and the likeliest alternatives of rows of logits, and the
// gradient of the first two.
//
//   m = max x, d = x - m, S = sum exp(scale d), T = sum scale d exp(scale d)
//   log p_v = scale d_v - log S,   entropy = log S - T / S
//   gradient: scale * (g_lp ([v = token] - p_v) - g_h p_v (log p_v + entropy))
//
// One pass over the logits.  A thread keeps (m, S, T) of its share and rescales when its maximum moves: with
// f = m - m' the sums become S 2^f and (T + S f) 2^f (everything in powers of two).  The maximum is a logit
// itself and is subtracted before anything is multiplied, so that neither a mask of the type's lowest value nor
// a row of nothing else overflows; a logit of -infinity adds 0.  Sums are fp32.
//
// The alternatives need no second pass: of the k largest thread maxima the smallest is a lower bound of the k-th largest
// logit.  Each thread also notes the maximum of every step, so that only the few steps that reach the bound are read again.
//
// Bound: the row's bytes.  A block takes a row; where there are too few rows to fill the card, a cluster of blocks
// takes one and joins its sums and alternatives through distributed shared memory.
#include <cooperative_groups.h>

#include <type_traits>

#include "score.cuh"

namespace cg = cooperative_groups;

namespace excp {
namespace {

constexpr int GRAD_BLOCK = 256;
constexpr int UNROLL = 4;                          // 16-byte loads in flight per thread
constexpr int TOP_MAX = 64;
constexpr int SLOTS = 16, OWNERS = 512;
constexpr int LIST = 1024;                         // candidates (or 8 blocks' alternatives) that are ranked at once
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float FAR = -200.f;                      // 2^FAR is 0 in fp32

__device__ __forceinline__ float exp2_fast(float x) {   // relative error 2^-22, subnormal results flushed to 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T> __host__ __device__ constexpr int per16() { return 16 / (int)sizeof(T); }
template <typename T>
__device__ __forceinline__ void unpack(const uint4& q, float* v) {
    const T* h = reinterpret_cast<const T*>(&q);
#pragma unroll
    for (int k = 0; k < per16<T>(); ++k) v[k] = wget(h, k);
}

// Two fp32 lanes per instruction.
__device__ __forceinline__ u64 pack2(float a, float b) { u64 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(u64 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ float low2(u64 v) { float a, b; unpack2(v, a, b); return a; }
__device__ __forceinline__ float high2(u64 v) { float a, b; unpack2(v, a, b); return b; }
__device__ __forceinline__ u64 add2(u64 a, u64 b) { u64 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ u64 mul2(u64 a, u64 b) { u64 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) { u64 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

struct Sums {
    float m, s, t;                                 // maximum logit, sum of 2^e, sum of e 2^e (e = scaled distance to m, base 2)
};
// The sums relative to a maximum m >= a.m.
__device__ __forceinline__ void move_to(Sums& a, float m, float c) {
    const float f = fmaxf((a.m - m) * c, FAR);
    const float e = exp2_fast(f);
    a.t = fmaf(a.s, f, a.t) * e;
    a.s *= e;
    a.m = m;
}

template <int N>
__device__ __forceinline__ float largest(const float (&v)[N]) {
    float top = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, v[k]);
    return top;
}
// The largest of 16-byte words of logits; two at a time where two fit 32 bits.
template <int U> __device__ __forceinline__ float largest_of(const uint4 (&q)[U], const float (&v)[U * 4], float) { return largest(v); }
template <int U, typename T>
__device__ __forceinline__ float largest_of(const uint4 (&q)[U], const float (&)[U * 8], T) {
    typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type T2;
    const T2* h = reinterpret_cast<const T2*>(q);
    T2 top = h[0];
#pragma unroll
    for (int k = 1; k < U * 4; ++k) top = __hmax2(top, h[k]);
    return fmaxf(wget(reinterpret_cast<const T*>(&top), 0), wget(reinterpret_cast<const T*>(&top), 1));
}

template <int N>
__device__ __forceinline__ void add_many(Sums& a, const float (&v)[N], float top, float c) {
    if (top > a.m) move_to(a, top, c);
    if (a.m == NEG_INF) {                          // nothing but -infinity so far (or NaN)
#pragma unroll
        for (int k = 0; k < N; ++k) if (v[k] != v[k]) a.s = v[k];
        return;
    }
    float s = 0.f, t = 0.f;
    if constexpr (N % 2 == 0) {
        const u64 m2 = pack2(-a.m, -a.m), c2 = pack2(c, c);
        u64 ss = 0, tt = 0;
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            const u64 e2 = mul2(add2(pack2(v[k], v[k + 1]), m2), c2);
            const u64 e = pack2(exp2_fast(low2(e2)), exp2_fast(high2(e2)));
            ss = add2(ss, e);
            tt = fma2(e2, e, tt);
        }
        s = low2(ss) + high2(ss);
        t = low2(tt) + high2(tt);
    }
    if (N == 1 || t != t) {                        // NaN also where a logit is -infinity: its distance times 0
        s = t = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float e2 = (v[k] - a.m) * c;
            const float e = exp2_fast(e2);         // a NaN logit stays NaN here
            s += e;
            t = fmaf(fmaxf(e2, FAR), e, t);
        }
    }
    a.s += s;
    a.t += t;
}

// Order of the alternatives: larger logit first, of equal ones the lower index; -0 counts as 0, NaN as largest.
__device__ __forceinline__ u32 value_key(float v) {
    if (v != v) return 0xffffffffu;
    const u32 b = __float_as_uint(v + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;   // never 0: -infinity gives 0x007fffff
}
__device__ __forceinline__ float key_value(u32 key) {      // the logit again (0 for -0)
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ u64 order_key(float v, u32 index) { return ((u64)value_key(v) << 32) | (0xffffffffu - index); }

// A block's share of a row: elements [lo, hi), of which [body, body + nvec * N) in whole 16-byte words.
template <typename T>
struct Share {
    const T* x;
    u32 lo, hi, body, nvec;
};
template <typename T>
__device__ __forceinline__ Share<T> share_of(const T* x, u32 vocab, u32 part, u32 parts) {
    constexpr u32 N = per16<T>();
    const u32 off = (u32)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (u32)sizeof(T);
    const u32 head = min(off, vocab);
    const u32 nvec = (vocab - head) / N;
    const u32 v0 = (u32)((u64)nvec * part / parts), v1 = (u32)((u64)nvec * (part + 1) / parts);
    return Share<T>{x, part == 0 ? 0 : head + v0 * N, part + 1 == parts ? vocab : head + v1 * N, head + v0 * N, v1 - v0};
}

template <int BLOCK>
struct Joint {                                     // shared memory of a block
    float m[BLOCK / 32], s[BLOCK / 32], t[BLOCK / 32];
    Sums sums;                                     // the block's
    alignas(16) unsigned short max_key[BLOCK];     // upper half of the keys of the thread maxima
    unsigned short step_key[SLOTS][BLOCK];         // the same of every slot (one or more steps) of every thread
    unsigned short owner[OWNERS];                  // slot << 8 | thread of the slots that hold candidates
    u32 bound, owners, count;
    u64 list[LIST];
    u64 best[TOP_MAX];                             // the block's alternatives, descending; 0 = none
    u64 warp_best[BLOCK / 32];
};

// Warp 0: a lower bound of the k-th largest logit of the share, as the upper 16 bits of its key (one bfloat16 step): the
// k-th largest of the thread maxima, found bit by bit.  0 where fewer than k threads have a maximum.
template <int BLOCK>
__device__ __forceinline__ u32 find_bound(const Joint<BLOCK>& j, u32 k) {
    constexpr int PAIRS = BLOCK / 64;
    u32 pair[PAIRS];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) pair[i] = reinterpret_cast<const u32*>(j.max_key)[threadIdx.x + 32 * i];
    u32 low = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
        const u32 test = low | (1u << bit);
        u32 n = 0;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) n += ((pair[i] & 0xffffu) >= test) + ((pair[i] >> 16) >= test);
        if (__reduce_add_sync(0xffffffffu, n) >= k) low = test;
    }
    return low;
}

// Writes the k largest of list[0..n) (distinct keys) to best[0..k), descending; 0 where there are fewer.
template <int BLOCK>
__device__ __forceinline__ void rank_list(Joint<BLOCK>& j, u32 n, u32 k) {
    for (u32 i = threadIdx.x; i < k; i += BLOCK) j.best[i] = 0;
    __syncthreads();
    for (u32 i = threadIdx.x; i < n; i += BLOCK) {
        const u64 mine = j.list[i];
        u32 rank = 0;
        for (u32 o = 0; o < n; ++o) rank += j.list[o] > mine;
        if (rank < k && mine) j.best[rank] = mine;
    }
    __syncthreads();
}

// The k largest of the share, one after another: where candidates outnumber the list (a row of equal logits), or a NaN
// keeps the thread maxima from saying anything.
template <typename T, int BLOCK>
__device__ void top_by_rounds(Joint<BLOCK>& j, const Share<T>& w, u32 k) {
    u64 last = ~0ull;
    for (u32 r = 0; r < k; ++r) {
        u64 mine = 0;
        for (u32 i = w.lo + threadIdx.x; i < w.hi; i += BLOCK) {
            const u64 key = order_key(wget(w.x, i), i);
            if (key < last && key > mine) mine = key;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const u64 other = __shfl_xor_sync(0xffffffffu, mine, o);
            if (other > mine) mine = other;
        }
        if ((threadIdx.x & 31) == 0) j.warp_best[threadIdx.x >> 5] = mine;
        __syncthreads();
        for (int i = 0; i < BLOCK / 32; ++i) if (j.warp_best[i] > mine) mine = j.warp_best[i];
        __syncthreads();
        if (threadIdx.x == 0) j.best[r] = mine;
        last = mine;
    }
    __syncthreads();
}

template <typename T, int BLOCK, bool CLUSTER>
__global__ void __launch_bounds__(BLOCK) logprobs_kernel(const T* __restrict__ logits, u32 vocab, u64 stride,
                                                         const long long* __restrict__ tokens, float scale, LogprobsOut out) {
    __shared__ Joint<BLOCK> j;
    constexpr u32 N = per16<T>();
    const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    u32 part = 0, parts = 1;
    if constexpr (CLUSTER) { part = cg::this_cluster().block_rank(); parts = cg::this_cluster().num_blocks(); }
    const u64 row = blockIdx.x / parts;
    const Share<T> w = share_of(logits + row * stride, vocab, part, parts);
    const float c = scale * LOG2E;
    long long token = -1;                          // the last thread writes the row's results
    float at_token = __uint_as_float(0x7fffffffu);
    if (part == 0 && tid == BLOCK - 1) {
        token = tokens[row];
        if (token >= 0 && token < (long long)vocab) at_token = wget(logits + row * stride, (u64)token);
    }

    // The body in UNROLL equal stretches; a step of the block takes BLOCK 16-byte words of each.
    const uint4* const body = reinterpret_cast<const uint4*>(w.x + w.body);
    const u32 stretch = (w.nvec + UNROLL - 1) / UNROLL;
    auto fetch = [&](uint4 (&q)[UNROLL][1], u32 p) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) if (p < stretch && u * stretch + p < w.nvec) q[u][0] = __ldg(body + u * stretch + p);
    };
    uint4 q[UNROLL][1];
    fetch(q, tid);
    // what lies before the first 16-byte word and behind the last
    const u32 tail = w.body + w.nvec * N;
    const bool has_head = w.lo + tid < w.body, has_tail = tail + tid < w.hi, any = has_head || has_tail || tid < stretch;
    const float head[1] = {has_head ? wget(w.x, w.lo + tid) : NEG_INF}, behind[1] = {has_tail ? wget(w.x, tail + tid) : NEG_INF};
    const u32 k = (u32)out.top;
    const u32 steps = (stretch + BLOCK - 1) / BLOCK, per_slot = (steps + SLOTS - 1) / SLOTS;
    if (tid == 0) j.owners = j.count = 0;

    Sums a{NEG_INF, 0.f, 0.f};
    if (has_head) add_many(a, head, head[0], c);
    if (has_tail) add_many(a, behind, behind[0], c);
    u32 slot = 0, left = per_slot;                 // steps that the slot still takes
    float slot_top = NEG_INF;
    for (u32 p = tid; p < stretch; p += BLOCK) {
        uint4 next[UNROLL][1];
        fetch(next, p + BLOCK);
        float top;
        if ((UNROLL - 1) * stretch + p < w.nvec) {
            float v[UNROLL * N];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) unpack<T>(q[u][0], v + u * N);
            top = largest_of(reinterpret_cast<const uint4 (&)[UNROLL]>(q), v, T());
            add_many(a, v, top, c);
        } else {
            top = NEG_INF;
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                if (u * stretch + p >= w.nvec) break;
                float v[N];
                unpack<T>(q[u][0], v);
                const float t = largest_of(q[u], v, T());
                add_many(a, v, t, c);
                top = fmaxf(top, t);
            }
        }
        if (k) {
            slot_top = fmaxf(slot_top, top);
            j.step_key[slot][tid] = (unsigned short)(value_key(slot_top) >> 16);
            if (--left == 0) { ++slot; left = per_slot; slot_top = NEG_INF; }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) q[u][0] = next[u][0];
    }
    if (k) j.max_key[tid] = (unsigned short)(any ? value_key(a.m) >> 16 : 0u);

    // join the threads: the maximum first, then sums relative to it
    float m = a.m;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) j.m[warp] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < BLOCK / 32; ++i) m = fmaxf(m, j.m[i]);
    if (k && warp == 0) {
        const u32 low = find_bound(j, k);
        if (lane == 0) j.bound = low;
    }
    if (m != NEG_INF) move_to(a, m, c);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
    }
    if (lane == 0) { j.s[warp] = a.s; j.t[warp] = a.t; }
    __syncthreads();
    a.s = a.t = 0.f;
#pragma unroll
    for (int i = 0; i < BLOCK / 32; ++i) { a.s += j.s[i]; a.t += j.t[i]; }
    a.m = m;

    if (k) {
        // the slots that reach the bound are read again, all their words at once, and their logits that reach it are ranked
        const u32 bound = j.bound;
        auto push = [&](float v, u32 i) {
            const u64 key = order_key(v, i);
            if ((u32)(key >> 48) < bound) return;
            const u32 at = atomicAdd(&j.count, 1u);
            if (at < LIST) j.list[at] = key;
        };
        for (u32 o = 0; tid + o * per_slot * BLOCK < stretch; ++o) {
            if (j.step_key[o][tid] < bound) continue;
            const u32 at = atomicAdd(&j.owners, 1u);
            if (at < OWNERS) j.owner[at] = (unsigned short)(o << 8 | tid);
        }
        if (has_head) push(head[0], w.lo + tid);
        if (has_tail) push(behind[0], tail + tid);
        __syncthreads();
        const u32 words = per_slot * UNROLL, total = min(j.owners, (u32)OWNERS) * words;
        for (u32 it = tid; it < total; it += BLOCK) {
            const u32 o = it / words, r = it - o * words, who = j.owner[o];
            const u32 p = (who & 255u) + ((who >> 8) * per_slot + r / UNROLL) * BLOCK, i = r % UNROLL * stretch + p;
            if (p >= stretch || i >= w.nvec) continue;
            const uint4 again = __ldg(body + i);
            float v[N];
            unpack<T>(again, v);
#pragma unroll
            for (u32 e = 0; e < N; ++e) push(v[e], w.body + i * N + e);
        }
        __syncthreads();
        if (a.s != a.s || j.owners > OWNERS || j.count > LIST) top_by_rounds(j, w, k);
        else rank_list(j, j.count, k);
    }
    if constexpr (CLUSTER) {
        cg::cluster_group cluster = cg::this_cluster();
        if (tid == 0) j.sums = a;
        cluster.sync();
        if (part == 0) {
            Sums all{NEG_INF, 0.f, 0.f};
            for (u32 i = 0; i < parts; ++i) all.m = fmaxf(all.m, cluster.map_shared_rank(&j, i)->sums.m);
            for (u32 i = 0; i < parts; ++i) {
                Sums b = cluster.map_shared_rank(&j, i)->sums;
                if (all.m != NEG_INF) move_to(b, all.m, c);
                all.s += b.s;
                all.t += b.t;
            }
            a = all;
            if (k) {
                for (u32 i = tid; i < parts * k; i += BLOCK) j.list[i] = cluster.map_shared_rank(&j, i / k)->best[i % k];
            }
        }
        cluster.sync();                            // the others' shared memory has been read
        if (part != 0) return;
        if (k) rank_list(j, parts * k, k);
    }

    const float log_s = logf(a.s);
    const bool empty = a.m == NEG_INF && a.s == 0.f;
    auto log_p = [&](float v) { return empty && v == v ? NEG_INF : fmaf(v - a.m, scale, -log_s); };
    if (tid == BLOCK - 1) {
        const float h = empty ? 0.f : fmaf(-LN2, a.t / a.s, log_s);
        out.logprob[row] = token < 0 ? 0.f : log_p(at_token);      // NaN for a token past the vocabulary
        if (out.entropy) out.entropy[row] = h;
        if (out.row_stats) reinterpret_cast<float4*>(out.row_stats)[row] = make_float4(a.m, a.s, h, 0.f);
    }
    for (u32 i = tid; i < k; i += BLOCK) {
        const u64 key = j.best[i];
        out.top_index[row * k + i] = 0xffffffffu - (u32)key;
        out.top_logprob[row * k + i] = log_p(key_value((u32)(key >> 32)));
    }
}

// p times a line in the distance: -scale p (g_lp + g_h (log p + entropy)), and scale g_lp at the token.
// A block takes UNROLL 16-byte words per thread of a row, counted from the row's first 16-byte boundary; the block
// of a row's first words also takes what lies before it.  VEC: each row of the gradient starts as far from a boundary as
// the logits' row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(GRAD_BLOCK) grad_kernel(const T* logits, u32 vocab, u64 stride, const long long* __restrict__ tokens,
                                                     float scale, const float* __restrict__ row_stats, const float* __restrict__ g_logprob,
                                                     const float* __restrict__ g_entropy, T* grad, u64 grad_stride, u32 chunks) {
    constexpr u32 N = per16<T>();
    const u64 row = blockIdx.x / chunks;
    const u32 chunk = blockIdx.x - (u32)row * chunks;
    const float4 st = __ldg(reinterpret_cast<const float4*>(row_stats) + row);
    const long long t = tokens[row];
    float gl = g_logprob && t >= 0 ? __ldg(g_logprob + row) : 0.f;
    if (t >= (long long)vocab) gl = __uint_as_float(0x7fffffffu);
    const float gh = g_entropy ? __ldg(g_entropy + row) : 0.f;
    const bool empty = st.x == NEG_INF && st.y == 0.f;
    const float c = scale * LOG2E, inv = scale / st.y;
    const float slope = -gh * LN2 * inv, base = -(gl + gh * (st.z - logf(st.y))) * inv, at_token = scale * gl;
    const T* x = logits + row * stride;
    T* y = grad + row * grad_stride;
    auto value = [&](float v, u32 i) {
        const float e2 = (v - st.x) * c;
        float r = exp2_fast(e2) * fmaf(fmaxf(e2, FAR), slope, base);
        if ((long long)i == t) r += at_token;
        return empty ? 0.f : r;
    };
    if (VEC) {
        const u32 head = min((u32)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (u32)sizeof(T), vocab);
        const u32 first = head + chunk * (GRAD_BLOCK * UNROLL * N);
        if (chunk == 0 && threadIdx.x < head) wput(y, threadIdx.x, value(wget(x, threadIdx.x), threadIdx.x));
        uint4 q[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const u32 i = first + (u * GRAD_BLOCK + threadIdx.x) * N;
            if (i + N <= vocab) q[u] = *reinterpret_cast<const uint4*>(x + i);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const u32 i = first + (u * GRAD_BLOCK + threadIdx.x) * N;
            if (i + N <= vocab) {
                float v[N];
                unpack<T>(q[u], v);
                uint4 r;
                T* h = reinterpret_cast<T*>(&r);
#pragma unroll
                for (u32 k = 0; k < N; ++k) wput(h, k, value(v[k], i + k));
                *reinterpret_cast<uint4*>(y + i) = r;
            } else {
                for (u32 k = 0; k < N && i + k < vocab; ++k) wput(y, i + k, value(wget(x, i + k), i + k));
            }
        }
    } else {
        const u32 first = chunk * (GRAD_BLOCK * UNROLL * N);
        const u32 end = min(vocab, first + GRAD_BLOCK * UNROLL * N);
        for (u32 i = first + threadIdx.x; i < end; i += GRAD_BLOCK) wput(y, i, value(wget(x, i), i));
    }
}

template <typename T, int BLOCK, bool CLUSTER>
void logprobs_launch(cudaStream_t s, const RowsIn& x, u32 parts, const long long* tokens, float scale, const LogprobsOut& out) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((u32)x.rows * parts);
    cfg.blockDim = dim3(BLOCK);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CLUSTER ? 1 : 0;
    cudaLaunchKernelEx(&cfg, logprobs_kernel<T, BLOCK, CLUSTER>, static_cast<const T*>(x.p), (u32)x.cols, x.stride, tokens, scale, out);
}

template <typename T>
void logprobs_as(int sms, cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const LogprobsOut& out) {
    // a cluster per row while rows leave SMs idle
    u32 parts = 1;
    while (parts < 8 && x.rows * parts * 2 <= (u64)sms) parts *= 2;
    if (parts > 1) logprobs_launch<T, 256, true>(s, x, parts, tokens, scale, out);
    else if (x.rows <= (u64)sms * 5) logprobs_launch<T, 256, false>(s, x, 1, tokens, scale, out);
    else logprobs_launch<T, 128, false>(s, x, 1, tokens, scale, out);
}

template <typename T>
void grad_as(cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const float* row_stats, const float* g_logprob,
             const float* g_entropy, T* grad, u64 grad_stride) {
    const T* p = static_cast<const T*>(x.p);
    const u32 chunk = GRAD_BLOCK * UNROLL * per16<T>(), chunks = (u32)((x.cols + chunk - 1) / chunk);
    const bool vec = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(grad)) & 15) == 0 &&
                     (x.rows == 1 || (((x.stride - grad_stride) * sizeof(T)) & 15) == 0);
    const u32 grid = (u32)x.rows * chunks;
    if (vec) grad_kernel<T, true><<<grid, GRAD_BLOCK, 0, s>>>(p, (u32)x.cols, x.stride, tokens, scale, row_stats, g_logprob, g_entropy, grad, grad_stride, chunks);
    else grad_kernel<T, false><<<grid, GRAD_BLOCK, 0, s>>>(p, (u32)x.cols, x.stride, tokens, scale, row_stats, g_logprob, g_entropy, grad, grad_stride, chunks);
}

}  // namespace

void launch_token_logprobs(int sms, cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const LogprobsOut& out) {
    if (x.dtype == DT_F32) logprobs_as<float>(sms, s, x, tokens, scale, out);
    else if (x.dtype == DT_F16) logprobs_as<__half>(sms, s, x, tokens, scale, out);
    else logprobs_as<__nv_bfloat16>(sms, s, x, tokens, scale, out);
}

void launch_token_logprobs_grad(int, cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const float* row_stats,
                                const float* g_logprob, const float* g_entropy, void* grad, u64 grad_stride) {
#define EXCP_G(T) grad_as<T>(s, x, tokens, scale, row_stats, g_logprob, g_entropy, static_cast<T*>(grad), grad_stride)
    if (x.dtype == DT_F32) EXCP_G(float);
    else if (x.dtype == DT_F16) EXCP_G(__half);
    else EXCP_G(__nv_bfloat16);
#undef EXCP_G
}

}  // namespace excp
