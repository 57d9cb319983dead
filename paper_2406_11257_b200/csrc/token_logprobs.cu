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
// The alternatives need no second pass.  With k of them wanted and W warps, each warp finds the ceil(k / W)-th largest of its
// threads' maxima; the smallest of these is a lower bound of the k-th largest logit.  Each thread also notes the maximum of
// every step, so that only the few steps that reach the bound are read again, and what reaches it is ranked.
//
// Bound at 16 bits: no unit by itself.  4096 x 32000 bf16 takes 50 us, with five alternatives 63-65; of the latter, issue alone
// would take 37 (10.5 instructions per logit), the exponentials 31 (16 per SM and cycle), the bytes 40.6 at the copy rate, and 63 %
// of the issue slots are taken.  78 registers a thread leave a third of the SM's warp slots filled: too few to overlap the three.
// At fp32 the bytes: 2048 x 50304 63 us (63.7).  One row of 50304 fp32 with twenty 8 us (latency).
// A block takes a row; where there are too few rows to fill the card, a cluster of blocks takes one and joins its sums and
// alternatives through distributed shared memory.  (Persistent blocks with a ring of chunks that bulk copies keep filled were
// slower, 4096 x 32000 bf16 58 us: what they hide is not what is missing.)
#include <cooperative_groups.h>

#include <type_traits>

#include "score_launch.cuh"

namespace cg = cooperative_groups;

namespace excp {
namespace {

constexpr int GRAD_BLOCK = 128;                    // (256: 2048 x 50304 bf16 66 us against 64, 5056 x 391 fp32 14 against 8.6)
constexpr int UNROLL = 4;                          // 16-byte loads in flight per thread
constexpr int TOP_MAX = 64;
constexpr int SLOTS = 16, OWNERS = 512;            // step maxima kept per thread; of them that are read again
constexpr int LIST = 512;                          // candidates (or 8 blocks' alternatives) that are ranked at once
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
    if (v != v) return 0xfffffffeu;                // above infinity, and no order key is ~0
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
    alignas(16) u64 list[LIST];
    u64 best[TOP_MAX];                             // the block's alternatives, descending; 0 = none
    u64 warp_best[BLOCK / 32];
    float m[BLOCK / 32], s[BLOCK / 32], t[BLOCK / 32];
    u32 warp_bound[BLOCK / 32];
    Sums sums;                                     // the block's
    u32 owners, count;                             // slots that hold candidates, candidates
    unsigned short step_key[SLOTS][BLOCK];         // upper half of the key of every slot's (one or more steps') maximum
    unsigned short owner[OWNERS];                  // slot << 8 | thread of the slots that hold candidates
};

// Rank of `mine` among list[0..n) (distinct keys).
template <int BLOCK>
__device__ __forceinline__ u32 rank_of(const Joint<BLOCK>& j, u64 mine, u32 n) {
    u32 rank = 0;
    u32 o = 0;
    for (; o + 8 <= n; o += 8) {
#pragma unroll
        for (u32 i = 0; i < 8; i += 2) {
            const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(j.list + o + i);
            rank += (two.x > mine) + (two.y > mine);
        }
    }
    for (; o < n; ++o) rank += j.list[o] > mine;
    return rank;
}

// The k largest of the share to best[], one after another: where candidates outnumber the list (a row of equal logits), or a NaN
// keeps the thread maxima from saying anything.
template <typename T, int BLOCK>
__device__ __noinline__ void top_by_rounds(Joint<BLOCK>& j, const T* x, u32 lo, u32 hi, u32 k) {
    u64 last = ~0ull;
    for (u32 r = 0; r < k; ++r) {
        u64 mine = 0;
        for (u32 i = lo + threadIdx.x; i < hi; i += BLOCK) {
            const u64 key = order_key(wget(x, i), i);
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

// What a thread holds of its share while it walks through it: a step of the block is U * BLOCK words, of which word
// u * BLOCK + thread is the thread's.
template <typename T, int BLOCK, int U>
struct Walk {
    static constexpr u32 N = (u32)per16<T>(), STEP = U * BLOCK;
    Share<T> w;
    Sums a{NEG_INF, 0.f, 0.f};
    float head, behind;                            // what lies before the first word and behind the last
    bool has_head, has_tail;
    u32 steps, per_slot, slot, left;
    float slot_top;

    __device__ __forceinline__ void start(const Share<T>& share, float c) {
        w = share;
        const u32 tid = threadIdx.x, tail = w.body + w.nvec * N;
        a = Sums{NEG_INF, 0.f, 0.f};
        has_head = w.lo + tid < w.body;
        has_tail = tail + tid < w.hi;
        head = has_head ? wget(w.x, w.lo + tid) : NEG_INF;
        behind = has_tail ? wget(w.x, tail + tid) : NEG_INF;
        steps = (w.nvec + STEP - 1) / STEP;
        per_slot = (steps + SLOTS - 1) / SLOTS;
        slot = 0;
        left = per_slot;
        slot_top = NEG_INF;
    }
    __device__ __forceinline__ u32 words(u32 step) const {       // the thread's words of a step
        const u32 first = step * STEP + threadIdx.x;
        return first >= w.nvec ? 0 : min((u32)U, (w.nvec - first + BLOCK - 1) / BLOCK);
    }
    __device__ __forceinline__ void take(const uint4 (&q)[U], u32 n, float c, bool keys, Joint<BLOCK>& j) {
        float top = NEG_INF;
        if (n == U) {
            float v[U * N];
#pragma unroll
            for (int u = 0; u < U; ++u) unpack<T>(q[u], v + u * N);
            top = largest_of(q, v, T());
            add_many(a, v, top, c);
        } else {
#pragma unroll
            for (u32 u = 0; u < U; ++u) {
                if (u >= n) break;
                const uint4 one[1] = {q[u]};
                float v[N];
                unpack<T>(q[u], v);
                const float t = largest_of(one, v, T());
                add_many(a, v, t, c);
                top = fmaxf(top, t);
            }
        }
        if (keys) {
            slot_top = fmaxf(slot_top, top);
            j.step_key[slot][threadIdx.x] = (unsigned short)(value_key(slot_top) >> 16);
            if (--left == 0) { ++slot; left = per_slot; slot_top = NEG_INF; }
        }
    }

    // Joins the block: a becomes its sums, and with k > 0 its alternatives are either in list[0..count), to be ranked, or (true)
    // in best[].
    __device__ __forceinline__ bool join(Joint<BLOCK>& j, u32 k, float c, u32& count) {
        constexpr u32 WARPS = BLOCK / 32;
        const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        if (has_head) { const float v[1] = {head}; add_many(a, v, head, c); }
        if (has_tail) { const float v[1] = {behind}; add_many(a, v, behind, c); }
        float m = a.m;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) j.m[warp] = m;
        // warps whose threads all have a word (the first ones)
        const u32 full = min(w.nvec, (u32)BLOCK) / 32, nth = full ? (k + full - 1) / full : 33;
        if (k && warp < full) {
            u32 key = value_key(a.m) >> 16, low = 0;
            for (u32 r = 0; r < nth && nth <= 32; ++r) {
                low = __reduce_max_sync(0xffffffffu, key);
                const u32 holds = __ballot_sync(0xffffffffu, key == low);
                if (lane == __ffs(holds) - 1) key = 0;
            }
            if (lane == 0) j.warp_bound[warp] = low;
        }
        __syncthreads();
#pragma unroll
        for (u32 i = 0; i < WARPS; ++i) m = fmaxf(m, j.m[i]);
        if (m != NEG_INF) move_to(a, m, c);
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
            a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
        }
        if (lane == 0) { j.s[warp] = a.s; j.t[warp] = a.t; }
        u32 bound = 0;                             // 0: everything is a candidate
        auto push = [&](float v, u32 i) {
            const u64 key = order_key(v, i);
            if ((u32)(key >> 48) < bound) return;
            const u32 at = atomicAdd(&j.count, 1u);
            if (at < LIST) j.list[at] = key;
        };
        const u32 tail = w.body + w.nvec * N;
        if (k) {
            if (nth <= 32) {
                bound = 0xffffu;
                for (u32 i = 0; i < full; ++i) bound = min(bound, j.warp_bound[i]);
            }
            for (u32 o = 0; (u64)o * per_slot * STEP + tid < w.nvec; ++o) {
                if (j.step_key[o][tid] < bound) continue;
                const u32 at = atomicAdd(&j.owners, 1u);
                if (at < OWNERS) j.owner[at] = (unsigned short)(o << 8 | tid);
            }
            if (has_head) push(head, w.lo + tid);
            if (has_tail) push(behind, tail + tid);
        }
        __syncthreads();
        a.s = a.t = 0.f;
#pragma unroll
        for (u32 i = 0; i < WARPS; ++i) { a.s += j.s[i]; a.t += j.t[i]; }
        a.m = m;
        if (!k) return false;
        // the slots that reach the bound are read again, all their words at once
        const uint4* body = reinterpret_cast<const uint4*>(w.x + w.body);
        const u32 owners = j.owners, per = per_slot * U, total = min(owners, (u32)OWNERS) * per;
        for (u32 it = tid; it < total; it += BLOCK) {
            const u32 o = it / per, r = it - o * per, who = j.owner[o];
            const u32 i = ((who >> 8) * per_slot * U + r) * BLOCK + (who & 255u);
            if (i >= w.nvec) continue;
            const uint4 again = __ldg(body + i);
            float v[N];
            unpack<T>(again, v);
#pragma unroll
            for (u32 e = 0; e < N; ++e) push(v[e], w.body + i * N + e);
        }
        __syncthreads();
        count = j.count;
        if (a.s == a.s && owners <= OWNERS && count <= LIST) return false;
        top_by_rounds<T, BLOCK>(j, w.x, w.lo, w.hi, k);
        return true;
    }
};

// The results of a row from its sums.
struct Row {
    float m, log_s, scale;
    bool empty;
    __device__ __forceinline__ Row(const Sums& a, float scale_) : m(a.m), log_s(logf(a.s)), scale(scale_), empty(a.m == NEG_INF && a.s == 0.f) {}
    __device__ __forceinline__ float log_p(float v) const { return empty && v == v ? NEG_INF : fmaf(v - m, scale, -log_s); }
    __device__ __forceinline__ void put(const LogprobsOut& out, u64 row, const Sums& a, long long token, float at_token) const {
        const float h = empty ? 0.f : fmaf(-LN2, a.t / a.s, log_s);
        out.logprob[row] = token < 0 ? 0.f : log_p(at_token);      // NaN for a token past the vocabulary
        if (out.entropy) out.entropy[row] = h;
        if (out.row_stats) reinterpret_cast<float4*>(out.row_stats)[row] = make_float4(a.m, a.s, h, 0.f);
    }
    __device__ __forceinline__ void put_top(const LogprobsOut& out, u64 row, u32 place, u64 key) const {
        out.top_index[row * out.top + place] = 0xffffffffu - (u32)key;
        out.top_logprob[row * out.top + place] = log_p(key_value((u32)(key >> 32)));
    }
};

template <typename T>
__device__ __forceinline__ float token_logit(const T* x, long long token, u32 vocab) {
    return token >= 0 && token < (long long)vocab ? wget(x, (u64)token) : __uint_as_float(0x7fffffffu);
}

template <typename T, int BLOCK, bool CLUSTER>
__global__ void __launch_bounds__(BLOCK, BLOCK == 128 ? 7 : 768 / BLOCK) logprobs_kernel(const T* __restrict__ logits, u32 vocab, u64 stride, const long long* __restrict__ tokens,
                                                      float scale, LogprobsOut out) {
    constexpr int U = 4;
    __shared__ Joint<BLOCK> j;
    wait_for_previous();
    let_next_start();
    u32 part = 0, parts = 1;
    if constexpr (CLUSTER) { part = cg::this_cluster().block_rank(); parts = cg::this_cluster().num_blocks(); }
    const u32 tid = threadIdx.x;
    const u64 row = blockIdx.x / parts;
    const float c = scale * LOG2E;
    const T* x = logits + row * stride;
    const u32 k = (u32)out.top;
    long long token = -1;                          // the last thread writes the row's results
    float at_token = 0.f;
    if (part == 0 && tid == BLOCK - 1) {
        token = tokens[row];
        at_token = token_logit(x, token, vocab);
    }
    if (tid == 0) j.owners = j.count = 0;
    for (u32 i = tid; i < k; i += BLOCK) j.best[i] = 0;
    Walk<T, BLOCK, U> walk;
    walk.start(share_of(x, vocab, part, parts), c);
    const uint4* const body = reinterpret_cast<const uint4*>(walk.w.x + walk.w.body);
    uint4 q[U];
    auto fetch = [&](uint4 (&to)[U], u32 step) {
#pragma unroll
        for (u32 u = 0; u < U; ++u) if (step * walk.STEP + u * BLOCK + tid < walk.w.nvec) to[u] = __ldg(body + step * walk.STEP + u * BLOCK + tid);
    };
    fetch(q, 0);
    for (u32 step = 0; step < walk.steps; ++step) {
        uint4 next[U];
        fetch(next, step + 1);
        const u32 n = walk.words(step);
        if (n) walk.take(q, n, c, k != 0, j);
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = next[u];
    }
    u32 count = 0;
    bool listed = !walk.join(j, k, c, count);
    Sums a = walk.a;
    if constexpr (CLUSTER) {
        cg::cluster_group cluster = cg::this_cluster();
        if (k && listed) {                         // the block's own alternatives in order
            for (u32 i = tid; i < count; i += BLOCK) {
                const u64 mine = j.list[i];
                const u32 rank = rank_of(j, mine, count);
                if (rank < k) j.best[rank] = mine;
            }
        }
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
            for (u32 i = tid; i < parts * k; i += BLOCK) j.list[i] = cluster.map_shared_rank(&j, i / k)->best[i % k];
        }
        cluster.sync();                            // the others' shared memory has been read
        if (part != 0) return;
        count = parts * k;
        listed = true;
    }
    const Row r(a, scale);
    if (tid == BLOCK - 1) r.put(out, row, a, token, at_token);
    if (listed) {
        for (u32 i = tid; k && i < count; i += BLOCK) {
            const u64 mine = j.list[i];
            const u32 rank = rank_of(j, mine, count);
            if (rank < k && mine) r.put_top(out, row, rank, mine);
        }
    } else {
        for (u32 i = tid; i < k; i += BLOCK) r.put_top(out, row, i, j.best[i]);
    }
}

// p times a line in the distance: -scale p (g_lp + g_h (log p + entropy)), and scale g_lp at the token.
// A block takes UNROLL 16-byte words per thread of a row, counted from the first 16-byte boundary of the gradient's row;
// the block of a row's first words also takes what lies before it.  SHIFT: the logits' row is not as far from such a
// boundary as the gradient's, and a word of logits is cut out of the two 16-byte words that hold it; the second is the
// next thread's first, so it comes from L1 (slack of 3 in 2048 x 50304 bf16: 82 us; value by value it was 162).
// The last rows come first: they are the ones that a preceding forward pass has left in L2; what is written goes past it.
// Bound: the bytes (2048 x 50304 bf16: 64 us, 6.4 TB/s).
template <typename T, bool SHIFT>
__global__ void __launch_bounds__(GRAD_BLOCK) grad_kernel(const T* logits, u64 rows, u32 vocab, u64 stride, const long long* __restrict__ tokens,
                                                     float scale, const float* __restrict__ row_stats, const float* __restrict__ g_logprob,
                                                     const float* __restrict__ g_entropy, T* grad, u64 grad_stride, u32 chunks) {
    constexpr u32 N = per16<T>();
    wait_for_previous();
    let_next_start();
    const u64 from_end = blockIdx.x / chunks, row = rows - 1 - from_end;
    const u32 chunk = blockIdx.x - (u32)from_end * chunks;
    const float4 st = __ldg(reinterpret_cast<const float4*>(row_stats) + row);
    const long long t = tokens[row];
    // nothing without g_logprob, whatever the token; NaN for one past the vocabulary
    const float gl = !g_logprob || t < 0 ? 0.f : t < (long long)vocab ? __ldg(g_logprob + row) : __uint_as_float(0x7fffffffu);
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
    const u32 head = min((u32)((16 - (reinterpret_cast<uintptr_t>(y) & 15)) & 15) / (u32)sizeof(T), vocab);
    const u32 first = head + chunk * (GRAD_BLOCK * UNROLL * N);
    if (chunk == 0 && threadIdx.x < head) wput(y, threadIdx.x, value(wget(x, threadIdx.x), threadIdx.x));
    // bytes from a 16-byte boundary to the logits that belong to a word of the gradient; the same for the whole row
    const u32 shift = SHIFT ? (u32)(reinterpret_cast<uintptr_t>(x + head) & 15) : 0u;
    uint4 q[UNROLL], after[SHIFT ? UNROLL : 1];
    bool whole[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const u32 i = first + (u * GRAD_BLOCK + threadIdx.x) * N;
        const char* p = reinterpret_cast<const char*>(x + i) - shift;
        // every byte that is read belongs to the row
        whole[u] = i + N <= vocab && (!SHIFT || (p >= reinterpret_cast<const char*>(x) && p + 32 <= reinterpret_cast<const char*>(x + vocab)));
        if (whole[u]) {
            q[u] = __ldcs(reinterpret_cast<const uint4*>(p));
            if (SHIFT) after[u] = __ldg(reinterpret_cast<const uint4*>(p) + 1);
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const u32 i = first + (u * GRAD_BLOCK + threadIdx.x) * N;
        if (whole[u]) {
            if (SHIFT) q[u] = cut16(q[u], after[u], shift);
            float v[N];
            unpack<T>(q[u], v);
            uint4 r;
            T* h = reinterpret_cast<T*>(&r);
#pragma unroll
            for (u32 k = 0; k < N; ++k) wput(h, k, value(v[k], i + k));
            __stcs(reinterpret_cast<uint4*>(y + i), r);
        } else {
            for (u32 k = 0; k < N && i + k < vocab; ++k) wput(y, i + k, value(wget(x, i + k), i + k));
        }
    }
}

template <typename T, int BLOCK, bool CLUSTER>
void logprobs_launch(cudaStream_t s, const RowsIn& x, u32 parts, const long long* tokens, float scale, const LogprobsOut& out) {
    launch_chained(logprobs_kernel<T, BLOCK, CLUSTER>, (u32)x.rows * parts, BLOCK, 0, CLUSTER ? parts : 0, s, static_cast<const T*>(x.p), (u32)x.cols,
                   x.stride, tokens, scale, out);
}

template <typename T>
void logprobs_as(int sms, cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const LogprobsOut& out) {
    // Few rows: 256 threads to a row, or a cluster of such blocks while rows leave SMs idle and each row is long enough to pay for
    // the cluster's two barriers (1 x 16000 bf16: 8 blocks 4.0 us, one 3.8; 1 x 32000: 4.2 and 4.7; 64 x 32000: 2 blocks 5.5,
    // one 4.8; 64 x 131072: 8.8 and 11.2).
    u32 parts = 1;
    while (parts < 8 && x.rows * parts * 2 <= (u64)sms) parts *= 2;
    if (parts > 1 && x.cols * parts >= 160 * 1024) logprobs_launch<T, 256, true>(s, x, parts, tokens, scale, out);
    else if (x.rows <= (u64)sms * 3 || (sizeof(T) == 2 && x.rows <= (u64)sms * 5 && x.cols > 16384)) logprobs_launch<T, 256, false>(s, x, 1, tokens, scale, out);
    // Many rows: blocks as small as registers last, so that while one joins its row others stream.  (4096 x 32000 bf16, five
    // alternatives: 96 threads 62 us, 128 65; 2048 x 50304 fp32: 128 threads 71 us, 96 74.  600 x 50304 bf16: 256
    // threads 22 us, 96 25; 600 x 4097: 9.3 and 6.5.)  Short ones: a warp to a row (5056 x 391 fp32: 10 us, 128 threads 19;
    // 4000 x 3000 bf16 15, 96 threads 19; 2000 x 8200 18 and 15); of up to 32 alternatives, each the maximum of a lane.
    else if (x.rows > (u64)sms * 8 && x.cols <= 4096 && out.top <= 32) logprobs_launch<T, 32, false>(s, x, 1, tokens, scale, out);
    else logprobs_launch<T, sizeof(T) == 2 ? 96 : 128, false>(s, x, 1, tokens, scale, out);
}

template <typename T, bool SHIFT>
void grad_launch(cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const float* row_stats, const float* g_logprob,
                 const float* g_entropy, T* grad, u64 grad_stride) {
    const u32 chunk = GRAD_BLOCK * UNROLL * per16<T>(), chunks = (u32)((x.cols + chunk - 1) / chunk);
    launch_chained(grad_kernel<T, SHIFT>, (u32)x.rows * chunks, GRAD_BLOCK, 0, 0, s, static_cast<const T*>(x.p), x.rows, (u32)x.cols, x.stride, tokens, scale,
                   row_stats, g_logprob, g_entropy, grad, grad_stride, chunks);
}
template <typename T>
void grad_as(cudaStream_t s, const RowsIn& x, const long long* tokens, float scale, const float* row_stats, const float* g_logprob,
             const float* g_entropy, T* grad, u64 grad_stride) {
    // every row of the logits as far from a 16-byte boundary as the gradient's
    const bool aligned = ((reinterpret_cast<uintptr_t>(x.p) ^ reinterpret_cast<uintptr_t>(grad)) & 15) == 0 &&
                         (x.rows == 1 || (((x.stride - grad_stride) * sizeof(T)) & 15) == 0);
    (aligned ? grad_launch<T, false> : grad_launch<T, true>)(s, x, tokens, scale, row_stats, g_logprob, g_entropy, grad, grad_stride);
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
