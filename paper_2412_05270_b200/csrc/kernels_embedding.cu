// Embedding lookup and its gradient: the first parameter of the model that the method does not project, whose
// gradient feeds apollo_adamw_step.
//
//   lookup    out[t] = scale E[index[t]]
//   gradient  dE[v]  = scale sum over {t : index[t] = v} of dOut[t]   (+ dE[v] when accumulating)
//
// A position whose index lies outside [0, rows) (padding) gives a zero row and no gradient.
//
// The gradient is a sum over positions grouped by token.  Positions are sorted by token (stable, so a token's
// positions stay in order), the sorted order is cut into windows of EMB_WINDOW positions, and a window sums the
// runs of equal tokens inside it in fp32: a run that is a token's whole segment is written at once, a piece of a
// longer segment goes to a partial row that embed_join_kernel adds up in window order.  A frequent token is so
// spread over the chip, and the order of every sum is a function of the indices alone: no float atomics, equal
// bits in every run.
#include "../../include/apollo.h"

#include <cooperative_groups.h>

#include <cmath>

#include "device_utils.cuh"
#include "host_utils.h"
#include "tc_ptx.cuh"

namespace cg = cooperative_groups;

namespace apollo {

namespace {

constexpr int EMB_THREADS = 256;
constexpr int EMB_WINDOW = 32;         // sorted positions per window
constexpr int SORT_THREADS = 512;
constexpr int SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_ITEMS = 8;          // keys per thread and tile
constexpr int SORT_TILE = SORT_THREADS * SORT_ITEMS;
constexpr int SORT_CLUSTER = 8;        // CTAs that share one sort through distributed shared memory
constexpr int SORT_BITS = 8, SORT_BINS = 1 << SORT_BITS;
constexpr size_t EMB_ALIGN = 256;

size_t emb_align(size_t x) { return (x + EMB_ALIGN - 1) / EMB_ALIGN * EMB_ALIGN; }

// Index t of the caller's array as a key in [0, rows]: everything outside [0, rows) becomes `rows`.
template <typename I>
__device__ __forceinline__ uint32_t index_key(const I* __restrict__ index, int64_t t, int64_t rows)
{
    const long long v = (long long)index[t];
    return v >= 0 && v < rows ? (uint32_t)v : (uint32_t)rows;
}

template <typename T> __device__ __forceinline__ void emb_store1(T* p, float v);
template <> __device__ __forceinline__ void emb_store1<float>(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void emb_store1<__nv_bfloat16>(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// 16 bytes: VEC elements of T
template <typename T> struct Vec16;
template <> struct Vec16<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void unpack(const uint4& r, float (&v)[4])
    {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&v)[4])
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Vec16<__nv_bfloat16> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void unpack(const uint4& r, float (&v)[8]) { unpack_bf16x8(r, v); }
    __device__ static __forceinline__ uint4 pack(const float (&v)[8])
    {
        return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
};

// The 16 bytes at p, wherever p lies: cut out of two aligned loads by a funnel shift per word, unless those would leave
// [first, last) (the row that p points into), where the elements are loaded one by one.
template <typename T>
__device__ __forceinline__ uint4 load16_anywhere(const T* p, const T* first, const T* last)
{
    const uint32_t mis = (uint32_t)((uintptr_t)p & 15u);
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) - mis);
    if (mis == 0) return __ldg(src);
    if (reinterpret_cast<uintptr_t>(src) < reinterpret_cast<uintptr_t>(first) || reinterpret_cast<uintptr_t>(src + 2) > reinterpret_cast<uintptr_t>(last)) {
        float v[Vec16<T>::N];
#pragma unroll
        for (int e = 0; e < Vec16<T>::N; ++e) v[e] = load1(p + e);
        return Vec16<T>::pack(v);
    }
    const uint4 lo = __ldg(src), hi = __ldg(src + 1);
    const uint32_t w[8] = { lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w };
    const uint32_t wsel = mis >> 2, sh = (mis & 2u) * 8u;
    uint32_t x[5];                                       // words wsel .. wsel + 4
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const uint32_t a = wsel & 1u ? w[i + 1] : w[i], b = wsel & 1u ? w[i + 3 < 8 ? i + 3 : 7] : w[i + 2];
        x[i] = wsel & 2u ? b : a;
    }
    return make_uint4(__funnelshift_r(x[0], x[1], sh), __funnelshift_r(x[1], x[2], sh), __funnelshift_r(x[2], x[3], sh), __funnelshift_r(x[3], x[4], sh));
}

// ---------------------------------------------------------------- lookup
// Bound: HBM, the distinct rows read once (repeats come from L2) and T x dim written.  `tpr` threads (a power of
// two) share a row; a thread has four vectors in flight.  VECTOR: table and output rows are whole aligned vectors.
// Else stores are vectors wherever the output row starts, the elements around them go one by one, and table rows at
// another offset are shifted into place (32768 x 2047 bf16: 76 us element by element, 46 us so; whole rows of 2048: 29).
template <typename T, typename I, bool VECTOR>
__global__ void __launch_bounds__(EMB_THREADS)
embed_kernel(const T* __restrict__ table, int64_t rows, int dim, const I* __restrict__ index, int64_t n_tokens, float scale,
             T* __restrict__ out, int64_t out_stride, int tpr_log2)
{
    const int tpr = 1 << tpr_log2, per_block = EMB_THREADS >> tpr_log2;
    const int lane = threadIdx.x & (tpr - 1), row_in_block = threadIdx.x >> tpr_log2;
    constexpr int V = Vec16<T>::N;
    for (int64_t t = (int64_t)blockIdx.x * per_block + row_in_block; t < n_tokens; t += (int64_t)gridDim.x * per_block) {
        const uint32_t key = index_key(index, t, rows);
        const bool live = key < rows;
        const T* src = table + (int64_t)key * dim;
        T* dst = out + t * out_stride;
        const int mis = VECTOR ? 0 : (int)(((uintptr_t)dst % 16) / sizeof(T));
        const int head = min(mis ? V - mis : 0, dim), vecs = (dim - head) / V;
        for (int u0 = lane; u0 < vecs; u0 += 4 * tpr) {
            uint4 raw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int u = u0 + k * tpr;
                raw[k] = make_uint4(0, 0, 0, 0);
                if (live && u < vecs) {
                    if constexpr (VECTOR) raw[k] = __ldg(reinterpret_cast<const uint4*>(src) + u);
                    else raw[k] = load16_anywhere(src + head + u * V, src, src + dim);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int u = u0 + k * tpr;
                if (u >= vecs) break;
                float v[V];
                Vec16<T>::unpack(raw[k], v);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] *= scale;
                __stcs(reinterpret_cast<uint4*>(dst + head) + u, Vec16<T>::pack(v));
            }
        }
        if constexpr (!VECTOR) {
            const int tail0 = head + vecs * V;
            if (lane < head) emb_store1<T>(dst + lane, live ? load1(src + lane) * scale : 0.0f);
            if (lane < dim - tail0) emb_store1<T>(dst + tail0 + lane, live ? load1(src + tail0 + lane) * scale : 0.0f);
        }
    }
}

// ---------------------------------------------------------------- sort (and zero fill beside it)
// Stable least-significant-digit radix sort of (token, position) by ONE cluster of SORT_CLUSTER CTAs; the other
// clusters of the launch write zeros over dE meanwhile (when not accumulating), which no step of the sort waits
// for: the sort costs no time as long as it is shorter than that fill (V dim e bytes of writes).
//
// A pass over one 8-bit digit: every CTA ranks its contiguous share and counts its digits; the counts are exchanged
// through distributed shared memory (base of a digit = all smaller digits anywhere + the same digit in CTAs of lower
// rank); then it scatters.  A share of more than one tile is counted first and ranked tile by tile after the exchange;
// one that fits a tile (SORT_CLUSTER x SORT_TILE = 32768 tokens) is read once.  Inside a tile a warp owns 32 x
// SORT_ITEMS consecutive keys (fewer in a share that does not fill the tile) and takes them 32 at a time: __match_any_sync gives the lanes with the same digit, the
// warp's running count of the digit the keys before them.
struct SortArgs {
    uint2* buf[2];          // (key, position) ping-pong
    int64_t n;
    int passes;
    uint32_t rows;          // sentinel key of positions without a row
};

template <typename I>
__global__ void __cluster_dims__(SORT_CLUSTER, 1, 1) __launch_bounds__(SORT_THREADS, 2)
embed_sort_kernel(const I* __restrict__ index, SortArgs a, uint4* __restrict__ zero, int64_t zero_vecs, char* __restrict__ zero_tail,
                  int zero_tail_bytes)
{
    ptx::grid_launch_dependents();
    if (blockIdx.x >= SORT_CLUSTER) {
        const int64_t stride = (int64_t)(gridDim.x - SORT_CLUSTER) * SORT_THREADS;
        const int64_t first = (int64_t)(blockIdx.x - SORT_CLUSTER) * SORT_THREADS + threadIdx.x;
        for (int64_t v = first; v < zero_vecs; v += stride) __stcs(zero + v, make_uint4(0, 0, 0, 0));
        if (first < zero_tail_bytes) zero_tail[first] = 0;
        return;
    }
    __shared__ uint32_t hist[2][SORT_BINS];              // this CTA's digit counts, read by the whole cluster; by pass parity
    __shared__ uint32_t base[SORT_BINS];                 // where the next key of a digit goes
    __shared__ uint32_t warp_hist[SORT_WARPS][SORT_BINS];
    __shared__ uint32_t scan[SORT_WARPS];
    cg::cluster_group cluster = cg::this_cluster();
    const int cta = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t share = (a.n + SORT_CLUSTER - 1) / SORT_CLUSTER;
    const int64_t begin = min((int64_t)cta * share, a.n), end = min(begin + share, a.n);
    const bool one_tile = share <= SORT_TILE;
    // keys of a warp, in rounds of 32: a short share is spread over all warps
    const int items = one_tile ? (int)((share + SORT_THREADS - 1) / SORT_THREADS) : SORT_ITEMS;

    uint2 kv[SORT_ITEMS];
    uint32_t rank[SORT_ITEMS];
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * SORT_BITS;
        const uint2* src = a.buf[(pass + 1) & 1];        // pass 0 reads the caller's indices
        uint2* dst = a.buf[pass & 1];
        uint32_t* const counts = hist[pass & 1];
        // ranks of a tile within its warp; warp_hist holds the warps' digit counts afterwards
        auto rank_tile = [&](int64_t tile) {
            for (int d = tid; d < SORT_BINS * SORT_WARPS; d += SORT_THREADS) (&warp_hist[0][0])[d] = 0;
            const int64_t first = tile + (int64_t)warp * (32 * items) + lane;
#pragma unroll
            for (int k = 0; k < SORT_ITEMS; ++k) {
                const int64_t t = k < items ? first + k * 32 : end;
                kv[k] = t >= end ? make_uint2(0xFFFFFFFFu, 0)
                                 : (pass == 0 ? make_uint2(index_key(index, t, (int64_t)a.rows), (uint32_t)t)
                                              : __ldcg(src + t));       // other CTAs wrote it in this launch: from L2
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < SORT_ITEMS; ++k) {
                if (k >= items) break;
                const bool valid = first + k * 32 < end;
                const uint32_t d = (kv[k].x >> shift) & (SORT_BINS - 1);
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, valid ? d : 0xFFFFFFFFu);
                const uint32_t below = __popc(same & ((1u << lane) - 1u));
                rank[k] = below;
                if (valid) rank[k] += warp_hist[warp][d];
                __syncwarp();
                if (valid && below == 0) warp_hist[warp][d] += __popc(same);
                __syncwarp();
            }
            __syncthreads();
        };
        // warp_hist -> exclusive sums over the warps; returns the digit's count (threads below SORT_BINS)
        auto scan_warps = [&](uint32_t run) {
#pragma unroll
            for (int w = 0; w < SORT_WARPS; ++w) {
                const uint32_t h = warp_hist[w][tid];
                warp_hist[w][tid] = run;
                run += h;
            }
            return run;
        };
        auto scatter = [&](int64_t tile, bool add_base) {
            const int64_t first = tile + (int64_t)warp * (32 * items) + lane;
#pragma unroll
            for (int k = 0; k < SORT_ITEMS; ++k)
                if (k < items && first + k * 32 < end) {
                    const uint32_t d = (kv[k].x >> shift) & (SORT_BINS - 1);
                    dst[warp_hist[warp][d] + rank[k] + (add_base ? base[d] : 0u)] = kv[k];
                }
        };
        if (one_tile) {
            rank_tile(begin);
            if (tid < SORT_BINS) counts[tid] = scan_warps(0);
        } else {
            for (int d = tid; d < SORT_BINS; d += SORT_THREADS) counts[d] = 0;
            __syncthreads();
            for (int64_t t = begin + tid; t < end; t += SORT_THREADS) {
                const uint32_t key = pass == 0 ? index_key(index, t, (int64_t)a.rows) : __ldcg(src + t).x;
                atomicAdd(&counts[(key >> shift) & (SORT_BINS - 1)], 1u);
            }
        }
        cluster.sync();
        // digit totals over the cluster, their exclusive sum, and the counts of this digit in CTAs before this one
        uint32_t total = 0, before = 0;
        if (tid < SORT_BINS) {
            uint32_t h[SORT_CLUSTER];
#pragma unroll
            for (int c = 0; c < SORT_CLUSTER; ++c) h[c] = cluster.map_shared_rank(counts, c)[tid];
#pragma unroll
            for (int c = 0; c < SORT_CLUSTER; ++c) {
                total += h[c];
                if (c < cta) before += h[c];
            }
        }
        uint32_t incl = total;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
            if (lane >= off) incl += up;
        }
        if (lane == 31) scan[warp] = incl;
        __syncthreads();
        if (tid < SORT_BINS) {
            uint32_t lower = 0;
            for (int w = 0; w < warp; ++w) lower += scan[w];
            base[tid] = lower + incl - total + before;
        }
        __syncthreads();
        if (one_tile) {
            scatter(begin, true);
        } else {
            for (int64_t tile = begin; tile < end; tile += SORT_TILE) {
                rank_tile(tile);
                if (tid < SORT_BINS) base[tid] = scan_warps(base[tid]);
                __syncthreads();
                scatter(tile, false);
                __syncthreads();
            }
        }
        __threadfence();
        cluster.sync();                                  // the other CTAs read what this one scattered, and have read its counts
    }
}

// ---------------------------------------------------------------- sums
// Columns [c, c + V) of dE row `row` <- acc (scaled), added to `old` when accumulating.
template <typename T, int V, bool ACCUMULATE>
__device__ __forceinline__ void grad_write(T* __restrict__ d_table, int64_t row, int dim, int c, const float (&acc)[V], float scale, const float (&old)[V])
{
    T* p = d_table + row * dim + c;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = ACCUMULATE ? fmaf(acc[e], scale, old[e]) : acc[e] * scale;
    if constexpr (V > 1) __stcs(reinterpret_cast<uint4*>(p), Vec16<T>::pack(v));
    else emb_store1<T>(p, v[0]);
}

// One window of sorted positions and `tpw` x V columns per thread group.  A run of equal tokens that both starts
// and ends in the window is written to dE; the first run, when it began in an earlier window, goes to partial row
// 2 w, and the last one, when it goes on in the next window, to partial row 2 w + 1 (a run that does both counts
// as the first).  (`sorted` is what the launch before wrote: no pointer here promises the compiler that it never
// changes, or a load could move ahead of the wait for that launch.)  Bound: HBM, every row of dOut read once; eight rows' loads are issued before the first is added.
template <typename T, bool VECTOR, bool ACCUMULATE>
__global__ void __launch_bounds__(EMB_THREADS, ACCUMULATE ? 2 : 4)
embed_sum_kernel(const T* __restrict__ d_out, int64_t out_stride, const uint2* sorted, int64_t n, uint32_t rows, int dim,
                 float scale, T* d_table, float* __restrict__ partial, int tpw_log2, int64_t windows)
{
    constexpr int V = VECTOR ? Vec16<T>::N : 1;
    __shared__ uint2 entry[EMB_THREADS / 8][EMB_WINDOW];
    const int tpw = 1 << tpw_log2, groups = EMB_THREADS >> tpw_log2;
    const int g = threadIdx.x >> tpw_log2, lane = threadIdx.x & (tpw - 1);
    ptx::grid_launch_dependents();
    ptx::grid_wait_previous();
    for (int i = threadIdx.x; i < groups * EMB_WINDOW; i += EMB_THREADS) {
        const int64_t at = ((int64_t)blockIdx.x * groups + i / EMB_WINDOW) * EMB_WINDOW + (i & (EMB_WINDOW - 1));
        entry[i / EMB_WINDOW][i & (EMB_WINDOW - 1)] = at < n ? sorted[at] : make_uint2(rows, 0);
    }
    __syncthreads();
    const int64_t w = (int64_t)blockIdx.x * groups + g;
    if (w >= windows) return;
    const int64_t at0 = w * EMB_WINDOW;
    const int count = (int)min((int64_t)EMB_WINDOW, n - at0);
    const bool from_before = at0 > 0 && sorted[at0 - 1].x == entry[g][0].x;
    const bool goes_on = at0 + EMB_WINDOW < n && sorted[at0 + EMB_WINDOW].x == entry[g][EMB_WINDOW - 1].x;
    for (int c = ((int)blockIdx.y * tpw + lane) * V; c < dim; c += (int)gridDim.y * tpw * V) {
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
        bool first_run = true;
        for (int i0 = 0; i0 < count; i0 += 8) {
            float v[8][V];
            uint4 raw[8];
            // what a run that ends here is added to: asked for with the rows, not when it is due
            uint4 old[ACCUMULATE && VECTOR ? 8 : 1];
            float old1[ACCUMULATE && !VECTOR ? 8 : 1];
            if constexpr (ACCUMULATE) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = i0 + k;
                    const uint32_t key = entry[g][i & (EMB_WINDOW - 1)].x;
                    const bool ends = i < count && key < rows && (i + 1 == count || entry[g][(i + 1) & (EMB_WINDOW - 1)].x != key);
                    const T* p = d_table + (int64_t)key * dim + c;
                    if constexpr (VECTOR) old[k] = ends ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
                    else old1[k] = ends ? load1(p) : 0.0f;
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool in = i0 + k < count && entry[g][(i0 + k) & (EMB_WINDOW - 1)].x < rows;
                const T* p = d_out + (int64_t)entry[g][(i0 + k) & (EMB_WINDOW - 1)].y * out_stride + c;
                if constexpr (VECTOR) raw[k] = in ? __ldcs(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
                else v[k][0] = in ? load1(p) : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + k;
                if (i >= count) break;
                if constexpr (VECTOR) Vec16<T>::unpack(raw[k], v[k]);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += v[k][e];
                const uint32_t key = entry[g][i].x;
                const bool last = i + 1 == count;
                if (!last && entry[g][i + 1].x == key) continue;
                if (key < rows) {
                    const bool piece_first = first_run && from_before, piece_last = last && goes_on;
                    if (piece_first || piece_last) {
                        float* p = partial + (2 * w + (piece_first ? 0 : 1)) * dim + c;
#pragma unroll
                        for (int e = 0; e < V; ++e) p[e] = acc[e];
                    } else {
                        float o[V];
                        if constexpr (ACCUMULATE) {
                            if constexpr (VECTOR) Vec16<T>::unpack(old[k], o);
                            else o[0] = old1[k];
                        }
                        grad_write<T, V, ACCUMULATE>(d_table, (int64_t)key, dim, c, acc, scale, o);
                    }
                }
                first_run = false;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.0f;
            }
        }
    }
}

// The segments that span windows: the blocks of the window in which such a segment starts add up its partial rows in
// window order, V columns per thread; a segment of many windows is shared by the block's warps, which take contiguous
// ranges of the windows and whose sums are added in warp order.  (V is 4 or 1: partial rows are whole vectors or not.)
constexpr int JOIN_SPLIT = 256;        // windows from which on a segment is shared (8192 positions of one token)

template <int V>
__device__ __forceinline__ void add_partial(float (&acc)[V], const float* p)
{
    if constexpr (V == 4) {
        const float4 x = *reinterpret_cast<const float4*>(p);
        acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
    } else {
        acc[0] += *p;
    }
}

template <typename T, int V, bool ACCUMULATE>
__global__ void __launch_bounds__(EMB_THREADS)
embed_join_kernel(const uint2* sorted, int64_t n, uint32_t rows, int dim, float scale, T* d_table, const float* partial)
{
    __shared__ float sums[EMB_THREADS / 32][32 * V];
    const int64_t w = blockIdx.x, next = (w + 1) * EMB_WINDOW;
    ptx::grid_wait_previous();
    const uint32_t key = sorted[next - 1].x, key_next = sorted[next].x, key_first = sorted[w * EMB_WINDOW].x;
    const uint32_t key_before = w > 0 ? sorted[w * EMB_WINDOW - 1].x : key_first;
    if (key >= rows || key_next != key) return;                  // nothing goes on into the next window
    if (w > 0 && key_first == key && key_before == key) return;  // it began earlier
    // the windows it reaches: those that begin with it, one behind the other (every thread looks at one)
    int64_t pieces = 1;                                          // window w holds partial row 2 w + 1, the later ones 2 x index
    for (int found = EMB_THREADS; found == EMB_THREADS; pieces += found) {
        const int64_t at = (w + pieces + threadIdx.x) * EMB_WINDOW;
        found = __syncthreads_count(at < n && sorted[at].x == key);
    }
    auto piece_at = [&](int64_t p) { return partial + (2 * (w + p) + (p == 0 ? 1 : 0)) * dim; };
    auto write = [&](int c, const float (&total)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float one[1] = { total[e] };
            float old[1] = { 0.0f };
            if constexpr (ACCUMULATE) old[0] = load1(d_table + (int64_t)key * dim + c + e);
            grad_write<T, 1, ACCUMULATE>(d_table, (int64_t)key, dim, c + e, one, scale, old);
        }
    };
    if (pieces <= JOIN_SPLIT) {
        for (int c = ((int)blockIdx.y * EMB_THREADS + threadIdx.x) * V; c < dim; c += (int)gridDim.y * EMB_THREADS * V) {
            float acc[V];
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.0f;
#pragma unroll 16
            for (int64_t p = 0; p < pieces; ++p) add_partial<V>(acc, piece_at(p) + c);
            write(c, acc);
        }
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t per = (pieces + EMB_THREADS / 32 - 1) / (EMB_THREADS / 32);
    const int64_t p0 = warp * per, p1 = min(p0 + per, pieces);
    for (int c0 = (int)blockIdx.y * 32 * V; c0 < dim; c0 += (int)gridDim.y * 32 * V) {
        const int c = c0 + lane * V;
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
        if (c < dim) {
#pragma unroll 8
            for (int64_t p = p0; p < p1; ++p) add_partial<V>(acc, piece_at(p) + c);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) sums[warp][lane * V + e] = acc[e];
        __syncthreads();
        if (warp == 0 && c < dim) {
            float total[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                total[e] = 0.0f;
                for (int k = 0; k < EMB_THREADS / 32; ++k) total[e] += sums[k][lane * V + e];
            }
            write(c, total);
        }
        __syncthreads();
    }
}

int log2_ceil(int64_t x)
{
    int b = 0;
    while (((int64_t)1 << b) < x) ++b;
    return b;
}

struct EmbLayout { size_t buf0, buf1, partial, total; };

EmbLayout embed_layout(int64_t n, int64_t dim)
{
    EmbLayout l;
    const int64_t windows = (n + EMB_WINDOW - 1) / EMB_WINDOW;
    l.buf0 = 0;
    l.buf1 = emb_align(sizeof(uint2) * (size_t)n);
    l.partial = 2 * l.buf1;
    l.total = l.partial + emb_align(sizeof(float) * 2 * (size_t)windows * (size_t)dim);
    if (l.total == 0) l.total = EMB_ALIGN;
    return l;
}

int check_embed(int64_t rows, int64_t dim, int32_t dtype, int32_t index_type, int64_t n, float scale, int64_t stride)
{
    if (dtype != APOLLO_DT_F32 && dtype != APOLLO_DT_BF16) return APOLLO_ERR_INVALID_ARG;
    if (index_type != APOLLO_INDEX_I32 && index_type != APOLLO_INDEX_I64) return APOLLO_ERR_INVALID_ARG;
    if (!std::isfinite(scale)) return APOLLO_ERR_INVALID_ARG;
    if (rows < 1 || dim < 1 || n < 0 || rows > INT32_MAX || dim > (int64_t)1 << 24 || n > INT32_MAX || stride < dim) return APOLLO_ERR_SHAPE;
    return APOLLO_OK;
}

template <typename T, typename I>
void run_embed(const void* table, int64_t rows, int dim, const void* index, int64_t n, float scale, void* out, int64_t stride, int sms, cudaStream_t stream)
{
    const bool vector = (size_t)dim * sizeof(T) % 16 == 0 && (size_t)stride * sizeof(T) % 16 == 0 &&
                        (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0;
    const int units = (dim + Vec16<T>::N - 1) / Vec16<T>::N;
    int lg = log2_ceil((units + 3) / 4);
    if (lg < 3) lg = 3;
    if (lg > 8) lg = 8;
    const int64_t blocks = (n + (EMB_THREADS >> lg) - 1) / (EMB_THREADS >> lg), most = 16LL * sms;
    const int grid = (int)(blocks < most ? blocks : most);
    if (vector) embed_kernel<T, I, true><<<grid, EMB_THREADS, 0, stream>>>((const T*)table, rows, dim, (const I*)index, n, scale, (T*)out, stride, lg);
    else embed_kernel<T, I, false><<<grid, EMB_THREADS, 0, stream>>>((const T*)table, rows, dim, (const I*)index, n, scale, (T*)out, stride, lg);
}

template <typename T, bool ACCUMULATE>
void run_embed_sum(const void* d_out, int64_t stride, const uint2* sorted, int64_t n, uint32_t rows, int dim, float scale,
                   void* d_table, float* partial, cudaStream_t stream)
{
    const bool vector = (size_t)dim * sizeof(T) % 16 == 0 && (size_t)stride * sizeof(T) % 16 == 0 &&
                        (uintptr_t)d_out % 16 == 0 && (uintptr_t)d_table % 16 == 0;
    const int units = vector ? dim / Vec16<T>::N : dim;
    int lg = log2_ceil(units);
    if (lg < 3) lg = 3;
    if (lg > 8) lg = 8;
    const int64_t windows = (n + EMB_WINDOW - 1) / EMB_WINDOW;
    const int groups = EMB_THREADS >> lg;
    const int cols = (units + (1 << lg) - 1) >> lg;
    const dim3 grid((unsigned)((windows + groups - 1) / groups), (unsigned)(cols < 1024 ? cols : 1024));
    launch_after(vector ? embed_sum_kernel<T, true, ACCUMULATE> : embed_sum_kernel<T, false, ACCUMULATE>, grid, dim3(EMB_THREADS), stream,
                 (const T*)d_out, stride, sorted, n, rows, dim, scale, (T*)d_table, partial, lg, windows);
    if (windows > 1) {
        const int v = dim % 4 == 0 ? 4 : 1;
        const int cb = (dim + EMB_THREADS * v - 1) / (EMB_THREADS * v);
        const dim3 jgrid((unsigned)(windows - 1), (unsigned)(cb < 64 ? cb : 64));
        launch_after(v == 4 ? embed_join_kernel<T, 4, ACCUMULATE> : embed_join_kernel<T, 1, ACCUMULATE>, jgrid, dim3(EMB_THREADS), stream,
                     sorted, n, rows, dim, scale, (T*)d_table, partial);
    }
}

}  // namespace

}  // namespace apollo

using namespace apollo;

extern "C" int apollo_embedding(const void* d_table, int64_t rows, int64_t dim, int32_t dtype, const void* d_index, int32_t index_type,
                                int64_t n_tokens, float scale, void* d_out, int64_t out_stride, void* cuda_stream)
{
    const int rc = check_embed(rows, dim, dtype, index_type, n_tokens, scale, out_stride);
    if (rc != APOLLO_OK) return rc;
    if (n_tokens == 0) return APOLLO_OK;
    if (!d_table || !d_index || !d_out) return APOLLO_ERR_INVALID_ARG;
    const size_t e = dtype == APOLLO_DT_BF16 ? 2 : 4, ie = index_type == APOLLO_INDEX_I64 ? 8 : 4;
    if ((uintptr_t)d_table % e || (uintptr_t)d_out % e || (uintptr_t)d_index % ie) return APOLLO_ERR_ALIGN;
    int sms = 0;
    const int drc = device_sms(&sms);
    if (drc != APOLLO_OK) return drc;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (dtype == APOLLO_DT_BF16) {
        if (index_type == APOLLO_INDEX_I64) run_embed<__nv_bfloat16, long long>(d_table, rows, (int)dim, d_index, n_tokens, scale, d_out, out_stride, sms, stream);
        else run_embed<__nv_bfloat16, int>(d_table, rows, (int)dim, d_index, n_tokens, scale, d_out, out_stride, sms, stream);
    } else {
        if (index_type == APOLLO_INDEX_I64) run_embed<float, long long>(d_table, rows, (int)dim, d_index, n_tokens, scale, d_out, out_stride, sms, stream);
        else run_embed<float, int>(d_table, rows, (int)dim, d_index, n_tokens, scale, d_out, out_stride, sms, stream);
    }
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}

extern "C" int apollo_embedding_grad_workspace_bytes(int64_t n_tokens, int64_t rows, int64_t dim, size_t* out_bytes)
{
    if (!out_bytes) return APOLLO_ERR_INVALID_ARG;
    const int rc = check_embed(rows, dim, APOLLO_DT_F32, APOLLO_INDEX_I32, n_tokens, 1.0f, dim);
    if (rc != APOLLO_OK) return rc;
    *out_bytes = embed_layout(n_tokens, dim).total;
    return APOLLO_OK;
}

extern "C" int apollo_embedding_grad(const void* d_out, int64_t out_stride, const void* d_index, int32_t index_type, int64_t n_tokens,
                                     int64_t rows, int64_t dim, int32_t dtype, float scale, int32_t accumulate, void* d_table_grad,
                                     void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    const int rc = check_embed(rows, dim, dtype, index_type, n_tokens, scale, out_stride);
    if (rc != APOLLO_OK) return rc;
    if ((accumulate != 0 && accumulate != 1) || !d_table_grad) return APOLLO_ERR_INVALID_ARG;
    const size_t e = dtype == APOLLO_DT_BF16 ? 2 : 4, ie = index_type == APOLLO_INDEX_I64 ? 8 : 4;
    if ((uintptr_t)d_table_grad % e || (uintptr_t)d_out % e || (uintptr_t)d_index % ie) return APOLLO_ERR_ALIGN;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const size_t bytes = (size_t)rows * (size_t)dim * e;
    if (n_tokens == 0) {
        if (!accumulate && cudaMemsetAsync(d_table_grad, 0, bytes, stream) != cudaSuccess) return APOLLO_ERR_CUDA;
        return APOLLO_OK;
    }
    if (!d_out || !d_index || !d_workspace) return APOLLO_ERR_INVALID_ARG;
    const EmbLayout l = embed_layout(n_tokens, dim);
    if ((uintptr_t)d_workspace % 16 || workspace_bytes < l.total) return APOLLO_ERR_WORKSPACE;
    int sms = 0;
    const int drc = device_sms(&sms);
    if (drc != APOLLO_OK) return drc;
    char* ws = static_cast<char*>(d_workspace);
    SortArgs a;
    a.buf[0] = reinterpret_cast<uint2*>(ws + l.buf0);
    a.buf[1] = reinterpret_cast<uint2*>(ws + l.buf1);
    a.n = n_tokens;
    a.rows = (uint32_t)rows;
    a.passes = (log2_ceil(rows + 1) + SORT_BITS - 1) / SORT_BITS;
    // zero fill: whole 16-byte vectors from the first 16-byte boundary on, the few bytes before and after by the tail threads
    char* z = static_cast<char*>(d_table_grad);
    int clusters = 1;
    int64_t vecs = 0;
    int tail = 0;
    char* tail_at = z;
    if (!accumulate) {
        if ((uintptr_t)z % 16) {
            if (cudaMemsetAsync(z, 0, bytes, stream) != cudaSuccess) return APOLLO_ERR_CUDA;
        } else {
            vecs = (int64_t)(bytes / 16);
            tail = (int)(bytes % 16);
            tail_at = z + vecs * 16;
            const int64_t want = (vecs + (int64_t)SORT_CLUSTER * SORT_THREADS * 8 - 1) / ((int64_t)SORT_CLUSTER * SORT_THREADS * 8);
            const int64_t most = 4LL * sms / SORT_CLUSTER;
            clusters += (int)(want < 1 ? 1 : want < most ? want : most);
        }
    }
    const dim3 grid((unsigned)(clusters * SORT_CLUSTER));
    if (index_type == APOLLO_INDEX_I64)
        embed_sort_kernel<long long><<<grid, SORT_THREADS, 0, stream>>>((const long long*)d_index, a, (uint4*)z, vecs, tail_at, tail);
    else
        embed_sort_kernel<int><<<grid, SORT_THREADS, 0, stream>>>((const int*)d_index, a, (uint4*)z, vecs, tail_at, tail);
    const uint2* sorted = a.buf[(a.passes - 1) & 1];
    float* partial = reinterpret_cast<float*>(ws + l.partial);
    const auto sum = dtype == APOLLO_DT_BF16 ? (accumulate ? run_embed_sum<__nv_bfloat16, true> : run_embed_sum<__nv_bfloat16, false>)
                                             : (accumulate ? run_embed_sum<float, true> : run_embed_sum<float, false>);
    sum(d_out, out_stride, sorted, n_tokens, (uint32_t)rows, (int)dim, scale, d_table_grad, partial, stream);
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}
