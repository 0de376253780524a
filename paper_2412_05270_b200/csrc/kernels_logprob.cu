// Log probabilities of given tokens with entropy and the best alternatives, and their gradient: the loss at the
// output head, whose weight the method does not project either.
//
//   z = scale * logit,  lse = log sum_j exp z_j,  logp = z_t - lse,  H = -sum_j p_j log p_j,  p_j = exp(z_j - lse)
//   d logit_j = scale (g (1[j = t] - p_j) - h p_j (z_j - lse + H))        for upstream g = d logp, h = d H
//
// Conventions: logits of -inf are masked words (p = 0, no gradient).  A row in which every word is masked has
// lse = -inf, logp = -inf, H = 0, no gradient.  A target outside [0, vocab) is ignored: logp = 0, g counts as 0.
//
// A log probability is formed as (logit - m) scale - log s, not as z - lse: lse is rounded at the size of the logits, and a
// common offset of them (1e4, say) must not cost the digits of a difference.
//
// Forward: one pass.  A thread keeps a reference m near the maximum of its elements and, with t = (logit - m) scale log2 e,
// s = sum 2^t and u = sum 2^t t; a new reference rescales both (u by the shift too).  Joined over the block, then over
// the cluster of CTAs that share a row, H = log s - log 2 u / s: the difference of small numbers, not of lse and a mean.
// Floor: HBM, N V e bytes; per element one exponential (16 a cycle and SM) and about five other instructions, which is
// why the sums run on packed pairs (fma.rn.f32x2) and the maximum of bfloat16 words is taken two at a time.  Measured: 8192 x
// 32000 bfloat16 119 us cold, 0.68 of the copy rate; neither memory nor issue is full (0.65 instructions a cycle and
// scheduler): the warps' cycles go to fixed latencies (19 %), the barriers at a row's end (17 %), the queue of the exponential unit
// (16 %), other warps' turns (15 %), and to memory 6 %.  fp32, 4096 x 32000: 95 us cold, 0.85.
#include "../../include/apollo.h"

#include <cooperative_groups.h>

#include <cmath>

#include "device_utils.cuh"
#include "host_utils.h"

namespace cg = cooperative_groups;

namespace apollo {

namespace {

constexpr int LP_MAX_TOP = APOLLO_MAX_TOP;
constexpr int LP_CAND = 1024;        // candidates one CTA collects before it falls back to picking one by one
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <typename T> struct LpVec;
template <> struct LpVec<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void unpack(const uint4& r, float (&v)[4])
    {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&v)[4])
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    __device__ static __forceinline__ void store1(float* p, float v) { *p = v; }
};
template <> struct LpVec<__nv_bfloat16> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void unpack(const uint4& r, float (&v)[8]) { unpack_bf16x8(r, v); }
    __device__ static __forceinline__ uint4 pack(const float (&v)[8])
    {
        return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
    __device__ static __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
};

// 2^x on the special-function unit (relative error about 2^-22; results below the normal range become 0)
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Pairs of floats in one 64-bit register.
__device__ __forceinline__ uint64_t pair2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Statistics of a set of logits v about a reference m (their maximum or a little less): s = sum 2^t, u = sum 2^t t, t = (v - m) L, L = scale log2 e.
struct Stat { float m, s, u; };

__device__ __forceinline__ Stat stat_empty() { return Stat{ -INFINITY, 0.0f, 0.0f }; }

// Moves st to the reference m >= st.m (m > -inf).
__device__ __forceinline__ void stat_shift(Stat& st, float m, float L)
{
    if (st.s != 0.0f) {                     // (a NaN s is != 0 and stays NaN)
        const float t = (st.m - m) * L, f = ex2(t);
        st.u = f * fmaf(fmaxf(t, -1000.0f), st.s, st.u);       // f is 0 long before the bound matters
        st.s *= f;
    }
    st.m = m;
}

__device__ __forceinline__ Stat stat_join(Stat a, Stat b, float L)
{
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return Stat{ m, a.s + b.s, a.u + b.u };   // nothing on either side (or NaN sums)
    stat_shift(a, m, L);
    stat_shift(b, m, L);
    return Stat{ m, a.s + b.s, a.u + b.u };
}

// Joins the statistics of N lanes (a power of two): the largest reference first, then plain sums.
template <int N>
__device__ __forceinline__ Stat stat_reduce(Stat st, float L)
{
    float m = st.m;
#pragma unroll
    for (int off = N / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
    if (m != -INFINITY) stat_shift(st, m, L);
#pragma unroll
    for (int off = N / 2; off > 0; off >>= 1) {
        st.s += __shfl_xor_sync(0xFFFFFFFFu, st.s, off);
        st.u += __shfl_xor_sync(0xFFFFFFFFu, st.u, off);
    }
    return st;
}

// A thread's running statistics, the sums in pairs.  The difference comes first, the factor L after it: masks of the
// type's lowest value are finite numbers whose multiples would overflow, and the maximum itself has t = 0 exactly.
struct Running {
    float m;
    uint64_t neg_m, s, u;                   // -m twice

    __device__ __forceinline__ void init() { m = -INFINITY; neg_m = s = u = 0ull; }
    __device__ __forceinline__ void raise(float top, float L)
    {
        if (m != -INFINITY || s != 0ull) {
            const float t = (m - top) * L, f = ex2(t);
            const uint64_t f2 = pair2(f, f), t2 = pair2(fmaxf(t, -1000.0f), fmaxf(t, -1000.0f));
            u = fma2(f2, fma2(t2, s, u), 0ull);
            s = fma2(f2, s, 0ull);
        }
        m = top;
        neg_m = pair2(-top, -top);
    }
    // Two logits.  2^t is 0 where t is -inf: keep the product with it 0.
    __device__ __forceinline__ void add(float v0, float v1, uint64_t L2)
    {
        float t0, t1;
        unpack2(mul2(add2(pair2(v0, v1), neg_m), L2), t0, t1);
        const uint64_t p = pair2(ex2(t0), ex2(t1));
        s = add2(s, p);
        u = fma2(p, pair2(fmaxf(t0, -1000.0f), fmaxf(t1, -1000.0f)), u);
    }
    __device__ __forceinline__ Stat stat() const
    {
        float s0, s1, u0, u1;
        unpack2(s, s0, s1);
        unpack2(u, u0, u1);
        return Stat{ m, s0 + s1, u0 + u1 };
    }
    // Makes room for logits up to `top` (NaN aside); false: nothing but -inf so far and among them.  The reference m is
    // moved only when a logit would exceed 2^8: any m near the maximum serves, and a warp rarely has to stop for it.
    __device__ __forceinline__ bool cover(float top, float L)
    {
        if ((top - m) * L > 8.0f) raise(top, L);      // (m = -inf: always, unless top is -inf too)
        return m != -INFINITY;
    }
    template <int N>
    __device__ __forceinline__ void add_all(const float (&v)[N], uint64_t L2)
    {
#pragma unroll
        for (int e = 0; e < N; e += 2) add(v[e], v[e + 1], L2);
    }
};

// The maximum of a 16-byte vector of logits (NaN aside), and a vector of nothing but masked words.
__device__ __forceinline__ float vec_max(const uint4& r, const __nv_bfloat16*)
{
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float vec_max(const uint4& r, const float*)
{
    return fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
}
__device__ __forceinline__ uint4 vec_masked(const __nv_bfloat16*) { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
__device__ __forceinline__ uint4 vec_masked(const float*) { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }

// Log probability of a logit v beside the statistics (m, log s); rounding must not make it positive.
__device__ __forceinline__ float log_prob(float v, float scale, float m, float log_s)
{
    const float d = v - m;
    // (masked words and differences that overflow: the products, whose difference may not)
    const float lp = isinf(d) ? __fmul_rn(v, scale) - fmaf(m, scale, log_s) : fmaf(d, scale, -log_s);
    return lp > 0.0f ? 0.0f : lp;
}

// Order of the alternatives: larger value first, then the lower index.  As one 64-bit key: the value's bits made
// monotone, then the complement of the index.  -0 counts as +0, NaN as the lowest value.  0 is "no entry".
__device__ __forceinline__ uint64_t top_key(float v, uint32_t index)
{
    uint32_t b = __float_as_uint(v + 0.0f);
    b = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    if (v != v) b = 1u;
    return ((uint64_t)b << 32) | (uint64_t)(~index);
}
__device__ __forceinline__ float top_value(uint64_t key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float((b & 0x80000000u) ? (b & 0x7FFFFFFFu) : ~b);
}

__device__ __forceinline__ uint64_t warp_max(uint64_t k)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, k, off);
        if (o > k) k = o;
    }
    return k;
}

struct LogprobArgs {
    const void* logits;
    const void* targets;
    int64_t stride, n_rows;
    int vocab, index64, top, parts;
    float scale;
    float* logprob;
    float* entropy;
    float* lse;
    float* top_logprob;
    int* top_index;
};

// A cluster of `parts` CTAs per row (1, 2, 4 or 8); each takes a contiguous part of the vocabulary, 4 vectors of 16
// bytes per thread and round, the few elements before the first 16-byte boundary and after the last beside them.
// The loads run a round ahead, and at the end of a row into the cluster's next row: its reduction costs no bandwidth.
//
// TOP: also the `top` best words, in the same pass.  After the first round the top-th largest of the threads' best keys
// is a lower bound of the top-th largest of all; from then on a thread looks at a vector's elements only if its maximum
// (which the statistics need anyway) reaches the bound, and collects those that do.  When the collection holds a few times
// `top` it is cut to its `top` best, which raises the bound.  Ranks are found by counting larger keys (they are distinct).  Should
// one round bring more than the collection holds (rising logits), the words are picked one by one from the row instead:
// slow, and right.
template <typename T, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, 768 / THREADS)
logprob_kernel(LogprobArgs a)
{
    constexpr int V = LpVec<T>::N, WARPS = THREADS / 32;
    __shared__ Stat part;                             // this CTA's statistics, read by rank 0 of the cluster
    __shared__ Stat warp_stat[WARPS];
    __shared__ uint64_t keys[TOP ? THREADS : 1];
    __shared__ uint64_t cand[TOP ? LP_CAND : 1];
    __shared__ uint64_t best[TOP ? LP_MAX_TOP : 1];   // this CTA's list, read by rank 0 of the cluster
    __shared__ uint64_t bound;
    __shared__ int n_cand;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = a.parts, rank = parts > 1 ? (int)cluster.block_rank() : 0;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per = ((a.vocab + parts - 1) / parts + V - 1) / V * V;
    const int begin = min(rank * per, a.vocab), end = min(begin + per, a.vocab);
    const float scale = a.scale, L = scale * LOG2E;
    const int64_t stride_rows = gridDim.x / parts;

    // where the vectors of a row's part lie
    struct Part { const T* row; const uint4* vec; int head, vecs, v0; };
    auto locate = [&](int64_t r) {
        Part p;
        p.row = static_cast<const T*>(a.logits) + r * a.stride;
        const int mis = (int)(((uintptr_t)(p.row + begin) % 16) / sizeof(T));
        p.head = min(mis ? V - mis : 0, end - begin);
        p.vecs = (end - begin - p.head) / V;
        p.v0 = begin + p.head;
        p.vec = reinterpret_cast<const uint4*>(p.row + p.v0);
        return p;
    };
    auto target_of = [&](int64_t r) {
        return a.index64 ? static_cast<const long long*>(a.targets)[r] : (long long)static_cast<const int*>(a.targets)[r];
    };
    int64_t r = blockIdx.x / parts;
    Part now = locate(r);
    uint4 next[4];                                    // beyond the last vector: masked words, which add nothing
    auto fetch = [&](int round) {
        const int u0 = round * 4 * THREADS + tid;
        if ((round + 1) * 4 * THREADS <= now.vecs) {
#pragma unroll
            for (int k = 0; k < 4; ++k) next[k] = __ldg(now.vec + u0 + k * THREADS);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) next[k] = u0 + k * THREADS < now.vecs ? __ldg(now.vec + u0 + k * THREADS) : vec_masked((const T*)nullptr);
        }
    };
    fetch(0);
    const uint64_t L2 = pair2(L, L);

    for (; r < a.n_rows; r += stride_rows) {
        const T* const row = now.row;
        const int vecs = now.vecs, v0 = now.v0, tail0 = v0 + vecs * V;
        // asked for at the start, used at the end
        const long long target = rank == 0 && tid == 0 ? target_of(r) : -1;
        const bool live = target >= 0 && target < a.vocab;
        const float chosen = live ? load1(row + target) : 0.0f;
        if constexpr (TOP) {
            if (tid == 0) { n_cand = 0; bound = 0; }
            if (tid < LP_MAX_TOP) best[tid] = 0;
        }
        Running run;
        run.init();
        // at most one element of the head and one of the tail per thread
        float edge[2] = { -INFINITY, -INFINITY };
        const int edge_at[2] = { tid < now.head ? begin + tid : -1, tid < end - tail0 ? tail0 + tid : -1 };
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (edge_at[i] >= 0) edge[i] = load1(row + edge_at[i]);

        uint64_t lim = 0;
        float lim_v = -INFINITY;
        bool flood = false;
        auto collect = [&](int i, float z) {
            const uint64_t k = top_key(z, (uint32_t)i);
            if (k < lim) return;
            const int at = atomicAdd(&n_cand, 1);
            if (at < LP_CAND) cand[at] = k;
        };
        // the `top` best of the collection, in order, to `best`
        auto cut = [&](int n) {
            for (int c = tid; c < n; c += THREADS) {
                const uint64_t k = cand[c];
                int ahead = 0;
#pragma unroll 8
                for (int o = 0; o < n; ++o) ahead += cand[o] > k ? 1 : 0;
                if (ahead < a.top) best[ahead] = k;
            }
            __syncthreads();
        };
        const int rounds = max(1, (vecs + 4 * THREADS - 1) / (4 * THREADS));
        for (int round = 0; round < rounds; ++round) {
            const int u0 = round * 4 * THREADS + tid;
            uint4 raw[4];
            float top[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) raw[k] = next[k];
            if (round + 1 < rounds) {
                fetch(round + 1);
            } else if (r + stride_rows < a.n_rows) {
                now = locate(r + stride_rows);
                fetch(0);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) top[k] = vec_max(raw[k], (const T*)nullptr);
            if (run.cover(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), L)) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v[V];
                    LpVec<T>::unpack(raw[k], v);
                    run.add_all(v, L2);
                }
            } else {
                // only masked words so far: or NaN
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v[V];
                    LpVec<T>::unpack(raw[k], v);
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (v[e] != v[e]) run.s = pair2(NAN, 0.0f);
                }
            }
            if constexpr (TOP) {
                if (round == 0) {
                    // the thread's best key: its largest value, found again at the lowest index
                    const float best_z = __fmul_rn(fmaxf(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), fmaxf(edge[0], edge[1])), scale);
                    int best_i = edge_at[1] >= 0 && __fmul_rn(edge[1], scale) == best_z ? edge_at[1] : -1;
#pragma unroll
                    for (int k = 3; k >= 0; --k) {
                        if (u0 + k * THREADS >= vecs || __fmul_rn(top[k], scale) != best_z) continue;
                        float v[V];
                        LpVec<T>::unpack(raw[k], v);
#pragma unroll
                        for (int e = V - 1; e >= 0; --e)
                            if (__fmul_rn(v[e], scale) == best_z) best_i = v0 + (u0 + k * THREADS) * V + e;
                    }
                    if (edge_at[0] >= 0 && __fmul_rn(edge[0], scale) == best_z) best_i = edge_at[0];
                    const uint64_t mine = best_i >= 0 ? top_key(best_z, (uint32_t)best_i) : 0;
                    // the top-th largest of the threads' keys (0 where fewer threads have one: then everything passes):
                    // every warp sorts its keys by counting, a key's place among all is then found by halving
                    keys[tid] = mine;
                    __syncwarp();
                    int in_warp = 0;
#pragma unroll 8
                    for (int k = 0; k < 32; ++k) {
                        const uint64_t o = keys[warp * 32 + k];
                        in_warp += o > mine || (o == 0 && mine == 0 && k < lane) ? 1 : 0;
                    }
                    __syncwarp();
                    keys[warp * 32 + in_warp] = mine;
                    __syncthreads();
                    int above = in_warp;
                    for (int w = 0; w < WARPS; ++w) {
                        if (w == warp) continue;
                        int lo = 0;                                     // keys of warp w larger than mine
#pragma unroll
                        for (int half = 16; half > 0; half >>= 1)
                            if (keys[w * 32 + lo + half - 1] > mine) lo += half;
                        if (lo == 31 && keys[w * 32 + 31] > mine) lo = 32;
                        above += lo;
                    }
                    if (mine != 0 && above == a.top - 1) bound = mine;
                    __syncthreads();
                    lim = bound;
                    lim_v = lim ? top_value(lim) : -INFINITY;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (edge_at[i] >= 0) collect(edge_at[i], __fmul_rn(edge[i], scale));
                }
                if (!flood) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (u0 + k * THREADS >= vecs) break;
                        if (__fmul_rn(top[k], scale) < lim_v) continue;
                        float v[V];
                        LpVec<T>::unpack(raw[k], v);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float z = __fmul_rn(v[e], scale);
                            if (!(z < lim_v)) collect(v0 + (u0 + k * THREADS) * V + e, z);
                        }
                    }
                    // whoever made the last entry has seen its count: all threads decide alike
                    if (__syncthreads_or(*reinterpret_cast<volatile int*>(&n_cand) > 3 * a.top + 32)) {
                        const int n = n_cand;
                        flood = n > LP_CAND;
                        if (!flood) {
                            cut(n);
                            if (tid < a.top) cand[tid] = best[tid];
                            if (tid == 0) n_cand = a.top;
                            lim = best[a.top - 1];
                            lim_v = top_value(lim);
                        }
                        __syncthreads();
                    }
                }
            }
        }
        if (run.cover(fmaxf(edge[0], edge[1]), L)) run.add_all(edge, L2);
        else if (edge[0] != edge[0] || edge[1] != edge[1]) run.s = pair2(NAN, 0.0f);
        const Stat st = stat_reduce<32>(run.stat(), L);
        if (lane == 0) warp_stat[warp] = st;
        __syncthreads();
        Stat all = stat_empty();
        if (warp == 0) {
            if (lane < WARPS) all = warp_stat[lane];
            all = stat_reduce<WARPS>(all, L);
            if (lane == 0) part = all;
        }
        if constexpr (TOP) {
            if (!flood) {
                cut(n_cand);
            } else {
                uint64_t last = ~0ull;
                for (int t = 0; t < a.top; ++t) {
                    uint64_t b = 0;
                    for (int i = begin + tid; i < end; i += THREADS) {
                        const uint64_t k = top_key(__fmul_rn(load1(row + i), scale), (uint32_t)i);
                        if (k < last && k > b) b = k;
                    }
                    b = warp_max(b);
                    __syncthreads();
                    if (lane == 0) keys[warp] = b;
                    __syncthreads();
                    for (int w = 0; w < WARPS; ++w) b = keys[w] > b ? keys[w] : b;
                    if (tid == 0) best[t] = b;
                    last = b;
                }
                __syncthreads();
            }
        }
        if (parts > 1) cluster.sync();
        if (rank == 0 && (TOP || warp == 0)) {
            if (TOP || parts > 1) {
                all = parts > 1 ? *cluster.map_shared_rank(&part, 0) : part;
                for (int c = 1; c < parts; ++c) all = stat_join(all, *cluster.map_shared_rank(&part, c), L);
            }
            const bool dead = __fmul_rn(all.m, scale) == -INFINITY && all.s == all.s;     // (and no NaN)
            const float log_s = dead ? 0.0f : logf(all.s);
            const float lse = dead ? -INFINITY : fmaf(all.m, scale, log_s);
            if (tid == 0) {
                a.lse[r] = lse;
                a.entropy[r] = dead ? 0.0f : log_s - LN2 * (all.u / all.s);
                a.logprob[r] = !live ? 0.0f : dead ? -INFINITY : log_prob(chosen, scale, all.m, log_s);
            }
            if constexpr (TOP) {
                const int n = parts * a.top;              // at most 8 x 32
                if (parts > 1) {
                    for (int c = tid; c < n; c += THREADS) cand[c] = cluster.map_shared_rank(best, c / a.top)[c % a.top];
                    __syncthreads();
                }
                for (int c = tid; c < n; c += THREADS) {
                    const uint64_t k = parts > 1 ? cand[c] : best[c];
                    int ahead = c;
                    if (parts > 1) {
                        ahead = 0;
                        for (int o = 0; o < n; ++o) ahead += cand[o] > k ? 1 : 0;
                    }
                    if (k != 0 && ahead < a.top) {
                        const int i = (int)~(uint32_t)k;
                        a.top_index[r * a.top + ahead] = i;
                        a.top_logprob[r * a.top + ahead] = dead ? -INFINITY : log_prob(load1(row + i), scale, all.m, log_s);
                    }
                }
            }
        }
        if (parts > 1) cluster.sync();                     // the other CTAs' shared memory has been read
        else __syncthreads();                              // this one's, before the next row
    }
}

struct LogprobGradArgs {
    const void* logits;
    const void* targets;
    int64_t stride, out_stride, n_rows;
    int vocab, index64;
    float scale;
    const float* lse;
    const float* entropy;
    const float* d_logprob;
    const float* d_entropy;      // may be null
    void* out;
};

constexpr int LG_THREADS = 256;

// One block per row and column chunk; reads the logits and writes their gradient, 2 e bytes an element: HBM-bound.
// Stores are 16-byte vectors whatever the row's alignment (the few elements around them go one by one).  Where the
// logits lie at another offset within 16 bytes, a vector is cut out of two aligned loads: a funnel shift per word.
// In place works: then both lie alike, and a thread writes what it has read.
template <typename T>
__global__ void __launch_bounds__(LG_THREADS)
logprob_grad_kernel(LogprobGradArgs a)
{
    constexpr int V = LpVec<T>::N;
    const int64_t r = blockIdx.x;
    const T* row = static_cast<const T*>(a.logits) + r * a.stride;
    T* out = static_cast<T*>(a.out) + r * a.out_stride;
    const int mis_out = (int)(((uintptr_t)out % 16) / sizeof(T));
    const int head = min(mis_out ? V - mis_out : 0, a.vocab), vecs = (a.vocab - head) / V, tail0 = head + vecs * V;
    const uint32_t mis = (uint32_t)((uintptr_t)(row + head) % 16);
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row + head) - mis);
    uint4* dst = reinterpret_cast<uint4*>(out + head);
    const int step = (int)gridDim.y * LG_THREADS, first = (int)blockIdx.y * LG_THREADS + (int)threadIdx.x;

    // the loads of the first round do not wait for the row's numbers
    uint4 raw[4];
    auto fetch = [&](int u0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int u = u0 + k * step;
            if (u >= vecs) break;
            if (mis == 0) {
                raw[k] = __ldcs(src + u);
            } else if (u > 0 && u + 1 < vecs) {
                const uint4 lo = __ldg(src + u), hi = __ldg(src + u + 1);
                const uint32_t w[8] = { lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w };
                const uint32_t wsel = mis >> 2, sh = (mis & 2u) * 8u;
                uint32_t x[5];                           // words wsel .. wsel + 4
#pragma unroll
                for (int i = 0; i < 5; ++i) {
                    const uint32_t p = wsel & 1u ? w[i + 1] : w[i], q = i + 3 < 8 ? (wsel & 1u ? w[i + 3] : w[i + 2]) : w[i + 2];
                    x[i] = wsel & 2u ? q : p;
                }
                raw[k] = make_uint4(__funnelshift_r(x[0], x[1], sh), __funnelshift_r(x[1], x[2], sh), __funnelshift_r(x[2], x[3], sh), __funnelshift_r(x[3], x[4], sh));
            } else {
                // the aligned loads of the first and the last vector could leave the row
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = load1(row + head + u * V + e);
                raw[k] = LpVec<T>::pack(v);
            }
        }
    };
    fetch(first);

    const long long t = a.index64 ? static_cast<const long long*>(a.targets)[r] : (long long)static_cast<const int*>(a.targets)[r];
    const bool live = t >= 0 && t < a.vocab;
    const float lse = a.lse[r], scale = a.scale;
    const float g = live ? a.d_logprob[r] : 0.0f, h = a.d_entropy ? a.d_entropy[r] : 0.0f;
    const bool dead = lse == -INFINITY;
    const float ent = a.entropy ? a.entropy[r] : 0.0f;
    const int at = live && !dead ? (int)t : -1;
    // -scale p (g + h (z - lse + H)) = p (k0 + k1 (z - lse))
    const float k1 = -scale * h, k0 = -scale * fmaf(h, ent, g), gs = scale * g;
    auto value = [&](float v) {
        const float d = __fmul_rn(v, scale) - lse;              // the z of the forward pass, rounded the same way
        const float p = ex2(d * LOG2E);
        return p == 0.0f || dead ? 0.0f : p * fmaf(k1, d, k0);
    };
    for (int u0 = first; u0 < vecs; u0 += 4 * step) {
        if (u0 != first) fetch(u0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int u = u0 + k * step;
            if (u >= vecs) break;
            float v[V];
            LpVec<T>::unpack(raw[k], v);
            const int hit = at - (head + u * V);                // the target's place in this vector, if it is here
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[e] = value(v[e]);
                if (e == hit) v[e] += gs;
            }
            __stcs(dst + u, LpVec<T>::pack(v));
        }
    }
    if (blockIdx.y == 0) {
        const int edge[2] = { (int)threadIdx.x < head ? (int)threadIdx.x : -1, tail0 + (int)threadIdx.x < a.vocab ? tail0 + (int)threadIdx.x : -1 };
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (edge[i] >= 0) LpVec<T>::store1(out + edge[i], value(load1(row + edge[i])) + (edge[i] == at ? gs : 0.0f));
    }
}

int check_rows(int64_t n_rows, int64_t vocab, int64_t stride, int32_t dtype, int32_t index_type, float scale)
{
    if (dtype != APOLLO_DT_F32 && dtype != APOLLO_DT_BF16) return APOLLO_ERR_INVALID_ARG;
    if (index_type != APOLLO_INDEX_I32 && index_type != APOLLO_INDEX_I64) return APOLLO_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || scale <= 0.0f) return APOLLO_ERR_INVALID_ARG;
    if (n_rows < 0 || vocab < 1 || n_rows > INT32_MAX / 8 || vocab > (int64_t)1 << 30 || stride < vocab) return APOLLO_ERR_SHAPE;
    return APOLLO_OK;
}

template <typename T, bool TOP, int THREADS>
cudaError_t launch_logprob(LogprobArgs a, int sms, cudaStream_t stream)
{
    // A row is shared by as many CTAs as keep the chip busy: up to 8 while there are fewer CTAs than SMs and every
    // CTA still has a few vectors per thread.
    a.parts = 1;
    while (a.parts < 8 && a.n_rows * a.parts * 2 <= sms && a.vocab / (a.parts * 2) >= 512) a.parts *= 2;
    const int64_t most = (int64_t)sms * 768 / THREADS;        // resident at once: they loop over the rows
    const int64_t rows = a.parts > 1 || a.n_rows < most ? a.n_rows : most;
    if (a.parts == 1) {
        logprob_kernel<T, TOP, THREADS><<<(unsigned)rows, THREADS, 0, stream>>>(a);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * a.parts));
    cfg.blockDim = dim3((unsigned)THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, logprob_kernel<T, TOP, THREADS>, a);
}

template <typename T>
cudaError_t run_logprob(const LogprobArgs& a, int sms, cudaStream_t stream)
{
    // short rows take small blocks: more rows at once, fewer idle threads
    if ((int64_t)a.vocab * (int64_t)sizeof(T) <= 8192)
        return a.top > 0 ? launch_logprob<T, true, 64>(a, sms, stream) : launch_logprob<T, false, 64>(a, sms, stream);
    return a.top > 0 ? launch_logprob<T, true, 256>(a, sms, stream) : launch_logprob<T, false, 256>(a, sms, stream);
}

template <typename T>
void run_logprob_grad(const LogprobGradArgs& a, cudaStream_t stream)
{
    const int units = a.vocab / LpVec<T>::N;
    int chunks = (units + 4 * LG_THREADS - 1) / (4 * LG_THREADS);
    if (chunks < 1) chunks = 1;
    if (chunks > 65535) chunks = 65535;
    logprob_grad_kernel<T><<<dim3((unsigned)a.n_rows, (unsigned)chunks), LG_THREADS, 0, stream>>>(a);
}

}  // namespace

}  // namespace apollo

using namespace apollo;

extern "C" int apollo_token_logprobs(const void* d_logits, int64_t row_stride, int64_t n_rows, int64_t vocab, int32_t dtype,
                                     const void* d_targets, int32_t index_type, float scale, int32_t top, float* d_logprob,
                                     float* d_entropy, float* d_lse, float* d_top_logprob, int32_t* d_top_index, void* cuda_stream)
{
    const int rc = check_rows(n_rows, vocab, row_stride, dtype, index_type, scale);
    if (rc != APOLLO_OK) return rc;
    if (top < 0 || top > APOLLO_MAX_TOP || top > vocab) return APOLLO_ERR_INVALID_ARG;
    if (n_rows == 0) return APOLLO_OK;
    if (!d_logits || !d_targets || !d_logprob || !d_entropy || !d_lse || (top > 0 && (!d_top_logprob || !d_top_index))) return APOLLO_ERR_INVALID_ARG;
    const size_t e = dtype == APOLLO_DT_BF16 ? 2 : 4, ie = index_type == APOLLO_INDEX_I64 ? 8 : 4;
    if ((uintptr_t)d_logits % e || (uintptr_t)d_targets % ie || (uintptr_t)d_logprob % 4 || (uintptr_t)d_entropy % 4 || (uintptr_t)d_lse % 4 ||
        (uintptr_t)d_top_logprob % 4 || (uintptr_t)d_top_index % 4)
        return APOLLO_ERR_ALIGN;
    int sms = 0;
    const int drc = device_sms(&sms);
    if (drc != APOLLO_OK) return drc;
    LogprobArgs a;
    a.logits = d_logits; a.targets = d_targets; a.stride = row_stride; a.n_rows = n_rows; a.vocab = (int)vocab;
    a.index64 = index_type == APOLLO_INDEX_I64; a.top = top; a.scale = scale;
    a.logprob = d_logprob; a.entropy = d_entropy; a.lse = d_lse; a.top_logprob = d_top_logprob; a.top_index = d_top_index;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t err = dtype == APOLLO_DT_BF16 ? run_logprob<__nv_bfloat16>(a, sms, stream) : run_logprob<float>(a, sms, stream);
    if (err != cudaSuccess) { cudaGetLastError(); return APOLLO_ERR_CUDA; }
    return APOLLO_OK;
}

extern "C" int apollo_token_logprobs_grad(const void* d_logits, int64_t row_stride, int64_t n_rows, int64_t vocab, int32_t dtype,
                                          const void* d_targets, int32_t index_type, float scale, const float* d_lse,
                                          const float* d_entropy, const float* d_grad_logprob, const float* d_grad_entropy,
                                          void* d_grad_logits, int64_t grad_stride, void* cuda_stream)
{
    int rc = check_rows(n_rows, vocab, row_stride, dtype, index_type, scale);
    if (rc != APOLLO_OK) return rc;
    if (grad_stride < vocab) return APOLLO_ERR_SHAPE;
    if (n_rows == 0) return APOLLO_OK;
    if (!d_logits || !d_targets || !d_lse || !d_grad_logprob || !d_grad_logits || (d_grad_entropy && !d_entropy)) return APOLLO_ERR_INVALID_ARG;
    if (d_grad_logits == d_logits && grad_stride != row_stride) return APOLLO_ERR_INVALID_ARG;
    const size_t e = dtype == APOLLO_DT_BF16 ? 2 : 4, ie = index_type == APOLLO_INDEX_I64 ? 8 : 4;
    if ((uintptr_t)d_logits % e || (uintptr_t)d_grad_logits % e || (uintptr_t)d_targets % ie || (uintptr_t)d_lse % 4 || (uintptr_t)d_entropy % 4 ||
        (uintptr_t)d_grad_logprob % 4 || (uintptr_t)d_grad_entropy % 4)
        return APOLLO_ERR_ALIGN;
    LogprobGradArgs a;
    a.logits = d_logits; a.targets = d_targets; a.stride = row_stride; a.out_stride = grad_stride; a.n_rows = n_rows; a.vocab = (int)vocab;
    a.index64 = index_type == APOLLO_INDEX_I64; a.scale = scale; a.lse = d_lse; a.entropy = d_grad_entropy ? d_entropy : nullptr;
    a.d_logprob = d_grad_logprob; a.d_entropy = d_grad_entropy; a.out = d_grad_logits;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (dtype == APOLLO_DT_BF16) run_logprob_grad<__nv_bfloat16>(a, stream);
    else run_logprob_grad<float>(a, stream);
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}
