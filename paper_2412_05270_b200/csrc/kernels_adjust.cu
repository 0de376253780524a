// Logits adjusted by penalties for repeated tokens, biases and grammar masks, and the gradient of that.
//
//   c_j, d_j = occurrences of word j in the row's history, and from position `start` on
//   x = logit_j;  c_j > 0: x <- x > 0 ? x / rho : x rho;  d_j > 0: x <- x - (phi d_j + pi);  x <- x + bias_j + named values;
//   mask bit 0: x <- -inf
//   a_j = allowed ? dout_j : 0;  dlogit_j = a_j {1, 1 / rho, rho};  dbias_j = a_j (summed over rows if shared);  dvalue_i = a_j
//
// A block of threads takes a chunk of the vocabulary for one row, or for a few rows in turn.  It counts the tokens of its chunk in a table in
// shared memory and lists the words that occur (integer atomics: their order decides the order of the list, not the results).  Then
// two passes: a stream over the whole chunk that knows of bias and mask alone, and the listed words once more, one a thread.  (With
// both in one pass, vectors looking into the table, nearly every warp of a training batch had a word to look up: 376 instructions
// a vector of eight instead of 40.)  Rows that share a history (the positions of a sequence in training) go on with the table of the row
// before: they add the tokens in between.  A table word holds
// [31] seen at all  [30..20] 1 + slot of the word's named value  [19..0] how often from `start` on.
#include "../../include/apollo.h"

#include <cmath>

#include "device_utils.cuh"
#include "host_utils.h"

namespace apollo {

namespace {

constexpr int AJ_THREADS = 256;
constexpr int AJ_UNITS = 4;              // vectors a thread has of a row's chunk at once
constexpr int AJ_BATCH = 4;              // loads a thread has in flight where they are scattered
constexpr int AJ_ROWS = 16;              // most rows in turn, without sums
constexpr uint32_t AJ_SEEN = 0x80000000u;
constexpr int AJ_SLOT_SHIFT = 20;
constexpr uint32_t AJ_COUNT = (1u << AJ_SLOT_SHIFT) - 1, AJ_SLOT = 0x7FFu;

struct Rules {
    const void* history;
    long long history_stride;
    long long share;                     // rows of logits per row of history
    int history_len;
    int history64, words64;
    const int* length;
    const int* start;
    const float *rho_at, *phi_at, *pi_at;
    float rho, phi, pi;
    const void* bias;
    long long bias_stride;
    const void* word;
    const float* value;
    int n_bias;
    const uint32_t* mask;
    long long mask_stride;
};

__device__ __forceinline__ int token_at(const void* p, long long i, int is64, int vocab)
{
    if (is64) {
        const long long v = static_cast<const long long*>(p)[i];
        return v >= 0 && v < vocab ? (int)v : -1;
    }
    const int v = static_cast<const int*>(p)[i];
    return v < vocab ? v : -1;
}

// The table of a chunk: `chunk` words, and the list of those that are not zero.
struct Table {
    uint32_t* word;
    uint16_t* list;                      // chunk <= 65536
    int* count;
    int j0, width;
    long long history = -1;              // what it holds: row of the history, tokens, first counted one
    int length = 0, start = 0;

    __device__ __forceinline__ Table(uint32_t* at, int* n, int chunk, int first, int w)
        : word(at), list(reinterpret_cast<uint16_t*>(at + chunk)), count(n), j0(first), width(w) {}
    static __host__ __device__ constexpr int words(int chunk, int entries) { return chunk + (entries + 1) / 2; }
    __device__ __forceinline__ void clear(int chunk)
    {
        for (int i = threadIdx.x * 4; i < chunk; i += AJ_THREADS * 4) *reinterpret_cast<uint4*>(word + i) = make_uint4(0, 0, 0, 0);
        if (threadIdx.x == 0) *count = 0;
    }
    __device__ __forceinline__ void append(int j) { list[atomicAdd(count, 1)] = (uint16_t)j; }
    // f(word, position) for the tokens of the chunk at positions [from, to).
    template <typename F>
    __device__ __forceinline__ void scan(const Rules& r, int vocab, int from, int to, F f)
    {
        const long long first = history * r.history_stride;
        for (int i = from + (int)threadIdx.x; i < to; i += AJ_THREADS * AJ_BATCH) {
            int j[AJ_BATCH];
#pragma unroll
            for (int k = 0; k < AJ_BATCH; ++k) {
                const int at = i + k * AJ_THREADS;
                j[k] = at < to ? token_at(r.history, first + at, r.history64, vocab) - j0 : -1;
            }
#pragma unroll
            for (int k = 0; k < AJ_BATCH; ++k) if (j[k] >= 0 && j[k] < width) f(j[k], i + k * AJ_THREADS);
        }
    }
    // The table of `row`, from that of the row before it where both have the same history.  Begins with a barrier; the caller ends with one.
    __device__ __forceinline__ void set(const Rules& r, long long row, int vocab, int chunk)
    {
        const long long mine = row / r.share;
        const int len = r.length ? min(max(r.length[row], 0), r.history_len) : r.history_len;
        const int from = r.start ? min(max(r.start[row], 0), len) : 0;
        __syncthreads();
        if (mine != history || len < length) {
            clear(chunk);
            __syncthreads();
            history = mine;
            length = start = 0;
        }
        // positions whose count begins or ends, among those the table has
        if (start < min(from, length)) scan(r, vocab, start, min(from, length), [&](int j, int) { atomicSub(word + j, 1u); });
        if (from < min(start, length)) scan(r, vocab, from, min(start, length), [&](int j, int) { atomicAdd(word + j, 1u); });
        scan(r, vocab, length, len, [&](int j, int i) {
            if (!(atomicOr(word + j, AJ_SEEN) & AJ_SEEN)) append(j);
            if (i >= from) atomicAdd(word + j, 1u);
        });
        length = len;
        start = from;
    }
};

// Sixteen bytes of a row: N elements.
template <typename T> struct Sixteen;
template <> struct Sixteen<float> {
    static constexpr int N = 4;
    using Entry = uint4;                 // of the table that makes 32-bit masks of mask bits, four bits at a time
    __device__ static __forceinline__ Entry entry(int bits) { return make_uint4(-(bits & 1), -(bits >> 1 & 1), -(bits >> 2 & 1), -(bits >> 3 & 1)); }
    __device__ static __forceinline__ uint4 masks(const Entry* t, uint32_t bits) { return t[bits]; }
    __device__ static __forceinline__ uint32_t minus_inf() { return 0xFF800000u; }
    __device__ static __forceinline__ void unpack(const uint4& w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static __forceinline__ uint4 gather(const float* p)
    {
        return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
    }
};
template <> struct Sixteen<__nv_bfloat16> {
    static constexpr int N = 8;
    using Entry = uint2;
    __device__ static __forceinline__ Entry entry(int bits)
    {
        return make_uint2((bits & 1) * 0xFFFFu | (bits >> 1 & 1) * 0xFFFF0000u, (bits >> 2 & 1) * 0xFFFFu | (bits >> 3 & 1) * 0xFFFF0000u);
    }
    __device__ static __forceinline__ uint4 masks(const Entry* t, uint32_t bits)
    {
        const uint2 a = t[bits & 15], b = t[bits >> 4];
        return make_uint4(a.x, a.y, b.x, b.y);
    }
    __device__ static __forceinline__ uint32_t minus_inf() { return 0xFF80FF80u; }
    __device__ static __forceinline__ void unpack(const uint4& w, float (&x)[8]) { unpack_bf16x8(w, x); }
    __device__ static __forceinline__ uint4 pack(const float (&x)[8])
    {
        return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
    __device__ static __forceinline__ uint4 gather(const __nv_bfloat16* p)
    {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
        return make_uint4(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16, q[4] | (uint32_t)q[5] << 16, q[6] | (uint32_t)q[7] << 16);
    }
};

__device__ __forceinline__ uint4 select4(const uint4& m, const uint4& w, uint32_t other)
{
    return make_uint4((w.x & m.x) | (other & ~m.x), (w.y & m.y) | (other & ~m.y), (w.z & m.z) | (other & ~m.z), (w.w & m.w) | (other & ~m.w));
}

// N mask bits from column j on.
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int j, int n_words)
{
    const int w = j >> 5, at = j & 31;
    const uint32_t lo = words[w], hi = at + N > 32 && w + 1 < n_words ? words[w + 1] : 0;
    return __funnelshift_r(lo, hi, at) & ((1u << N) - 1u);
}
__device__ __forceinline__ bool allowed(const uint32_t* words, int j) { return !words || (words[j >> 5] >> (j & 31) & 1u); }

// A chunk of a row cut at the 16-byte boundaries of `out`: `full` vectors from column `first` on, the columns before and behind one by one.
template <typename T>
struct Span {
    static constexpr int N = Sixteen<T>::N;
    int first, full, head, tail;
    __device__ __forceinline__ Span(const T* out, int j0, int width)
    {
        head = min((int)((16 - ((uintptr_t)(out + j0) & 15)) % 16 / sizeof(T)), width);
        first = j0 + head;
        full = (width - head) / N;
        tail = width - head - full * N;
    }
    // the column that this thread has apart from the vectors, or -1 (N <= 8: lanes of the first two warps)
    __device__ __forceinline__ int single() const
    {
        const int t = threadIdx.x;
        return t < head ? first - head + t : t >= 32 && t - 32 < tail ? first + full * N + t - 32 : -1;
    }
};
template <typename T>
__device__ __forceinline__ bool on_boundary(const T* row, int first) { return ((uintptr_t)(row + first) & 15) == 0; }
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p, bool aligned)
{
    return aligned ? *reinterpret_cast<const uint4*>(p) : Sixteen<T>::gather(p);
}

struct AdjustArgs {
    const void* logits;
    void* out;
    long long stride, out_stride, n_rows;
    int vocab, chunk, chunks, rows;      // rows: in turn
    int entries;                         // of the list at most
    Rules r;
};

// TABLE: there is a history or there are named values.
template <typename T, bool TABLE>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_kernel(const __grid_constant__ AdjustArgs a)
{
    using S = Sixteen<T>;
    constexpr int N = S::N;
    extern __shared__ __align__(16) uint32_t shared[];
    __shared__ typename S::Entry masks[16];
    __shared__ int listed;
    if (threadIdx.x < 16) masks[threadIdx.x] = S::entry((int)threadIdx.x);
    if constexpr (!TABLE) __syncthreads();             // (otherwise there will be one)
    const int part = blockIdx.x % a.chunks;
    const long long begin = (long long)(blockIdx.x / a.chunks) * a.rows, end = min(begin + a.rows, a.n_rows);
    const int j0 = part * a.chunk, width = min(a.chunk, a.vocab - j0), mask_words = (a.vocab + 31) / 32;
    Table table(shared, &listed, a.chunk, j0, width);
    float* sums = reinterpret_cast<float*>(shared + Table::words(a.chunk, a.entries));
    int* words = reinterpret_cast<int*>(sums + a.r.n_bias);
    const bool place = a.logits == a.out, sparse = place && !a.r.bias;
    for (long long row = begin; row < end; ++row) {
        const T* const x0 = static_cast<const T*>(a.logits) + row * a.stride;
        T* const y0 = static_cast<T*>(a.out) + row * a.out_stride;
        const T* const b0 = a.r.bias ? static_cast<const T*>(a.r.bias) + row * a.r.bias_stride : nullptr;
        const uint32_t* const m0 = a.r.mask ? a.r.mask + row * a.r.mask_stride : nullptr;
        const Span<T> span(y0, j0, width);
        const bool x_aligned = on_boundary(x0, span.first), b_aligned = b0 && on_boundary(b0, span.first);
        // read before the table is there
        uint4 ahead[AJ_UNITS];
        if (!sparse) {
#pragma unroll
            for (int q = 0; q < AJ_UNITS; ++q) {
                const int u = q * AJ_THREADS + threadIdx.x;
                if (u < span.full) ahead[q] = load16(x0 + span.first + u * N, x_aligned);
            }
        }
        float rho = 1.0f, phi = 0.0f, pi = 0.0f;
        // the word's logit with everything that concerns it
        auto adjusted = [&](int j) {
            const uint32_t t = table.word[j];
            float x = (float)x0[j0 + j];
            if (t & (AJ_SEEN | AJ_COUNT)) x = x > 0.0f ? __fdiv_rn(x, rho) : x * rho;
            if (t & AJ_COUNT) x -= fmaf(phi, (float)(t & AJ_COUNT), pi);
            if (b0) x += (float)b0[j0 + j];
            const uint32_t slot = t >> AJ_SLOT_SHIFT & AJ_SLOT;
            return slot ? x + sums[slot - 1] : x;
        };
        if constexpr (TABLE) {
            for (int i = threadIdx.x; i < a.r.n_bias; i += AJ_THREADS) words[i] = token_at(a.r.word, row * a.r.n_bias + i, a.r.words64, a.vocab);
            if (a.r.history) {
                rho = a.r.rho_at ? a.r.rho_at[row] : a.r.rho;
                phi = a.r.phi_at ? a.r.phi_at[row] : a.r.phi;
                pi = a.r.pi_at ? a.r.pi_at[row] : a.r.pi;
                table.set(a.r, row, a.vocab, a.chunk);
            } else {
                table.clear(a.chunk);
            }
            if (a.r.n_bias) {                          // (such rows are not taken in turn)
                __syncthreads();
                // the first pair of a word sums the values of all its pairs, in order
                for (int i = threadIdx.x; i < a.r.n_bias; i += AJ_THREADS) {
                    const int w = words[i];
                    if (w < j0 || w >= j0 + width) continue;
                    bool first = true;
                    for (int k = 0; k < i && first; ++k) first = words[k] != w;
                    if (!first) continue;
                    float sum = 0.0f;
                    for (int k = i; k < a.r.n_bias; ++k) if (words[k] == w) sum += a.r.value[row * a.r.n_bias + k];
                    sums[i] = sum;
                    if (atomicOr(table.word + (w - j0), (uint32_t)(i + 1) << AJ_SLOT_SHIFT) == 0) table.append(w - j0);
                }
            }
            if (place && b0) {                         // the logits will be gone: results go to the table (such rows are not taken in turn either)
                __syncthreads();
                for (int i = threadIdx.x; i < listed; i += AJ_THREADS) {
                    const int j = table.list[i];
                    table.word[j] = __float_as_uint(adjusted(j));
                }
                __syncthreads();
            }
        }
        if (!sparse) {
#pragma unroll
            for (int q = 0; q < AJ_UNITS; ++q) {
                const int u = q * AJ_THREADS + threadIdx.x, j = span.first + u * N;
                if (u >= span.full) break;
                uint4 w = ahead[q];
                if (b0) {
                    float x[N], b[N];
                    S::unpack(w, x);
                    S::unpack(load16(b0 + j, b_aligned), b);
#pragma unroll
                    for (int e = 0; e < N; ++e) x[e] += b[e];
                    w = S::pack(x);
                }
                if (m0) w = select4(S::masks(masks, bits_at<N>(m0, j, mask_words)), w, S::minus_inf());
                *reinterpret_cast<uint4*>(y0 + j) = w;
            }
        } else if (m0) {
            for (int u = threadIdx.x; u < span.full; u += AJ_THREADS) {
                const int j = span.first + u * N;
                const uint32_t live = bits_at<N>(m0, j, mask_words);
                if (live == (1u << N) - 1u) continue;
                uint4* const y = reinterpret_cast<uint4*>(y0 + j);
                *y = select4(S::masks(masks, live), live ? *y : make_uint4(0, 0, 0, 0), S::minus_inf());
            }
        }
        if (const int j = span.single(); j >= 0) {
            if (!allowed(m0, j)) y0[j] = (T)-INFINITY;
            else if (!sparse) y0[j] = (T)(b0 ? (float)x0[j] + (float)b0[j] : (float)x0[j]);
        }
        if constexpr (TABLE) {
            __syncthreads();
            const int n = listed;
            for (int i = threadIdx.x; i < n; i += AJ_THREADS * AJ_BATCH) {
                float y[AJ_BATCH];
                int at[AJ_BATCH];
#pragma unroll
                for (int k = 0; k < AJ_BATCH; ++k) {
                    const int j = i + k * AJ_THREADS < n ? table.list[i + k * AJ_THREADS] : -1;
                    at[k] = j >= 0 && allowed(m0, j0 + j) ? j0 + j : -1;
                    if (at[k] >= 0) y[k] = place && b0 ? __uint_as_float(table.word[j]) : adjusted(j);
                }
#pragma unroll
                for (int k = 0; k < AJ_BATCH; ++k) if (at[k] >= 0) y0[at[k]] = (T)y[k];
            }
        }
    }
}

struct AdjustGradArgs {
    const void* logits;
    const void* dout;
    void* dlogits;
    void* dbias;                         // rows of its own (dbias_stride > 0), or null
    float* partial;                      // shared bias: sums over the rows of a block of threads, vocab floats each
    float* dvalue;
    long long stride, dout_stride, dlogits_stride, dbias_stride, n_rows;
    int vocab, chunk, chunks, rows;
    Rules r;
};

__device__ __forceinline__ void store_partial(float* p, float a, float b, float c, float d) { p[0] = a; p[1] = b; p[2] = c; p[3] = d; }

// SUM: the sums over the rows stay in registers.  Every row's vectors have to start at the same columns then; where they do not,
// WIDE = false takes the columns one by one.
template <typename T, bool TABLE, bool SUM, bool WIDE>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_grad_kernel(const __grid_constant__ AdjustGradArgs a)
{
    using S = Sixteen<T>;
    constexpr int N = WIDE ? S::N : 1;
    extern __shared__ __align__(16) uint32_t shared[];
    __shared__ typename S::Entry masks[16];
    __shared__ int listed;
    if (threadIdx.x < 16) masks[threadIdx.x] = S::entry((int)threadIdx.x);
    if constexpr (!TABLE) __syncthreads();             // (otherwise there will be one)
    const int part = blockIdx.x % a.chunks;
    const long long group = blockIdx.x / a.chunks, begin = group * a.rows, end = min(begin + a.rows, a.n_rows);
    const int j0 = part * a.chunk, width = min(a.chunk, a.vocab - j0), mask_words = (a.vocab + 31) / 32;
    Table table(shared, &listed, a.chunk, j0, width);
    const bool place = a.dlogits == a.dout;
    const bool sparse = place && !SUM && !a.dbias;
    float sum[SUM ? AJ_UNITS : 1][N], edge = 0.0f;
#pragma unroll
    for (int q = 0; q < (SUM ? AJ_UNITS : 1); ++q)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[q][e] = 0.0f;
    for (long long row = begin; row < end; ++row) {
        const T* const x0 = static_cast<const T*>(a.logits) + row * a.stride;
        const T* const g0 = static_cast<const T*>(a.dout) + row * a.dout_stride;
        T* const y0 = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
        T* const b0 = a.dbias ? static_cast<T*>(a.dbias) + row * a.dbias_stride : nullptr;
        const uint32_t* const m0 = a.r.mask ? a.r.mask + row * a.r.mask_stride : nullptr;
        const Span<T> span(y0, j0, width);
        const bool g_aligned = on_boundary(g0, span.first), b_aligned = b0 && on_boundary(b0, span.first);
        // read before the table is there
        uint4 ahead[WIDE ? AJ_UNITS : 1];
        if constexpr (WIDE) {
            if (!sparse) {
#pragma unroll
                for (int q = 0; q < AJ_UNITS; ++q) {
                    const int u = q * AJ_THREADS + threadIdx.x;
                    if (u < span.full) ahead[q] = load16(g0 + span.first + u * N, g_aligned);
                }
            }
        }
        float rho = 1.0f;
        if constexpr (TABLE) {
            rho = a.r.rho_at ? a.r.rho_at[row] : a.r.rho;
            table.set(a.r, row, a.vocab, a.chunk);
        }
        if (a.dvalue) {
            // (in place: before anything of the row is overwritten)
            for (int i = threadIdx.x; i < a.r.n_bias; i += AJ_THREADS) {
                const int w = token_at(a.r.word, row * a.r.n_bias + i, a.r.words64, a.vocab);
                if (w < 0 ? j0 == 0 : w >= j0 && w < j0 + width) a.dvalue[row * a.r.n_bias + i] = w >= 0 && allowed(m0, w) ? (float)g0[w] : 0.0f;
            }
            if (place) __syncthreads();
        }
        auto column = [&](int j, float& total) {
            const float g = allowed(m0, j) ? (float)g0[j] : 0.0f;
            if constexpr (SUM) total += g;
            if (b0) b0[j] = (T)g;
            y0[j] = (T)g;
        };
        if constexpr (!WIDE) {
#pragma unroll
            for (int q = 0; q < AJ_UNITS; ++q) {
                const int u = q * AJ_THREADS + threadIdx.x;
                if (u < width) column(j0 + u, sum[q][0]);
            }
        } else {
            if (!sparse) {
#pragma unroll
                for (int q = 0; q < AJ_UNITS; ++q) {
                    const int u = q * AJ_THREADS + threadIdx.x, j = span.first + u * N;
                    if (u >= span.full) break;
                    uint4 w = ahead[q];
                    if (m0) w = select4(S::masks(masks, bits_at<N>(m0, j, mask_words)), w, 0);
                    if constexpr (SUM) {
                        float g[N];
                        S::unpack(w, g);
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[q][e] += g[e];
                    }
                    if (b0) {
                        if (b_aligned) {
                            *reinterpret_cast<uint4*>(b0 + j) = w;
                        } else {
                            float g[N];
                            S::unpack(w, g);
#pragma unroll
                            for (int e = 0; e < N; ++e) b0[j + e] = (T)g[e];
                        }
                    }
                    if (!place || m0) *reinterpret_cast<uint4*>(y0 + j) = w;
                }
            } else if (m0) {
                for (int u = threadIdx.x; u < span.full; u += AJ_THREADS) {
                    const int j = span.first + u * N;
                    const uint32_t live = bits_at<N>(m0, j, mask_words);
                    if (live == (1u << N) - 1u) continue;
                    uint4* const y = reinterpret_cast<uint4*>(y0 + j);
                    *y = select4(S::masks(masks, live), live ? *y : make_uint4(0, 0, 0, 0), 0);
                }
            }
            if (const int j = span.single(); j >= 0) column(j, edge);
        }
        if constexpr (TABLE) {
            __syncthreads();
            const int n = listed;
            for (int i = threadIdx.x; i < n; i += AJ_THREADS * AJ_BATCH) {
                float g[AJ_BATCH], x[AJ_BATCH];
                int at[AJ_BATCH];
#pragma unroll
                for (int k = 0; k < AJ_BATCH; ++k) {
                    const int w = i + k * AJ_THREADS < n ? j0 + table.list[i + k * AJ_THREADS] : -1;
                    at[k] = w >= 0 && allowed(m0, w) ? w : -1;
                    if (at[k] >= 0) { g[k] = (float)g0[w]; x[k] = (float)x0[w]; }
                }
#pragma unroll
                for (int k = 0; k < AJ_BATCH; ++k)
                    if (at[k] >= 0) y0[at[k]] = (T)(x[k] > 0.0f ? __fdiv_rn(g[k], rho) : g[k] * rho);
            }
        }
    }
    if constexpr (SUM) {
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q) {
            const int u = (q * AJ_THREADS + (int)threadIdx.x) * N;
            if (WIDE && u + N <= width) {
#pragma unroll
                for (int e = 0; e < N; e += 4)
                    if constexpr (N >= 4) store_partial(a.partial + group * a.vocab + j0 + u + e, sum[q][e], sum[q][e + 1], sum[q][e + 2], sum[q][e + 3]);
            } else if (!WIDE && u < width) {
                a.partial[group * a.vocab + j0 + u] = sum[q][0];
            }
        }
        // (wide rows start on a boundary: the columns left are behind the last whole vector)
        if (WIDE && threadIdx.x >= 32 && (int)threadIdx.x - 32 < width % N) a.partial[group * a.vocab + j0 + width / N * N + threadIdx.x - 32] = edge;
    }
}

template <typename T>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_bias_join_kernel(const float* __restrict__ partial, int groups, int vocab, T* __restrict__ dbias)
{
    const int j = blockIdx.x * AJ_THREADS + threadIdx.x;
    if (j >= vocab) return;
    float sum = 0.0f;
    for (int g = 0; g < groups; ++g) sum += partial[(long long)g * vocab + j];
    dbias[j] = (T)sum;
}

constexpr int AJ_MAX_GROUPS = 256;       // rows of partial sums for a shared bias
constexpr int AJ_PLACE_CHUNK = 16384;    // in place: little is read, so more words for one reading of the history
constexpr int AJ_MOST_SMEM = (Table::words(AJ_PLACE_CHUNK, AJ_PLACE_CHUNK) + 2 * APOLLO_MAX_BIAS_WORDS) * 4;

bool whole_vectors(const void* p, int64_t stride, size_t e) { return (uintptr_t)p % 16 == 0 && (size_t)stride * e % 16 == 0; }

int check_rules(const apollo_logit_rules* r, int64_t n_rows, int64_t vocab, size_t e, bool gradient, Rules* out)
{
    Rules q = {};
    q.share = 1; q.rho = 1.0f;
    if (r->d_history) {
        if ((r->history_type != APOLLO_INDEX_I32 && r->history_type != APOLLO_INDEX_I64) || r->history_rows < 1 || r->history_len < 0 ||
            r->history_stride < 0)
            return APOLLO_ERR_INVALID_ARG;
        if (r->history_len > APOLLO_MAX_HISTORY || n_rows % r->history_rows || (r->history_stride > 0 && r->history_stride < r->history_len))
            return APOLLO_ERR_SHAPE;
        if (!r->d_repetition && !(r->repetition > 0.0f && std::isfinite(r->repetition))) return APOLLO_ERR_INVALID_ARG;
        if (!gradient && ((!r->d_frequency && !std::isfinite(r->frequency)) || (!r->d_presence && !std::isfinite(r->presence)))) return APOLLO_ERR_INVALID_ARG;
        if ((uintptr_t)r->d_history % (r->history_type == APOLLO_INDEX_I64 ? 8 : 4) || (uintptr_t)r->d_length % 4 || (uintptr_t)r->d_start % 4 ||
            (uintptr_t)r->d_repetition % 4 || (uintptr_t)r->d_frequency % 4 || (uintptr_t)r->d_presence % 4)
            return APOLLO_ERR_ALIGN;
        q.history = r->d_history; q.history_stride = r->history_stride; q.share = n_rows / r->history_rows; q.history_len = (int)r->history_len;
        q.history64 = r->history_type == APOLLO_INDEX_I64;
        q.length = r->d_length; q.start = r->d_start;
        q.rho_at = r->d_repetition; q.phi_at = r->d_frequency; q.pi_at = r->d_presence;
        q.rho = r->repetition; q.phi = r->frequency; q.pi = r->presence;
    }
    if (r->d_bias && !gradient) {
        if (r->bias_stride != 0 && r->bias_stride < vocab) return APOLLO_ERR_SHAPE;
        if ((uintptr_t)r->d_bias % e) return APOLLO_ERR_ALIGN;
        q.bias = r->d_bias; q.bias_stride = r->bias_stride;
    }
    if (r->n_bias < 0 || (r->n_bias > 0 && (!r->d_bias_word || (!gradient && !r->d_bias_value)))) return APOLLO_ERR_INVALID_ARG;
    if (r->n_bias > APOLLO_MAX_BIAS_WORDS) return APOLLO_ERR_SHAPE;
    if (r->n_bias > 0) {
        if (r->bias_word_type != APOLLO_INDEX_I32 && r->bias_word_type != APOLLO_INDEX_I64) return APOLLO_ERR_INVALID_ARG;
        if ((uintptr_t)r->d_bias_word % (r->bias_word_type == APOLLO_INDEX_I64 ? 8 : 4) || (uintptr_t)r->d_bias_value % 4) return APOLLO_ERR_ALIGN;
        q.word = r->d_bias_word; q.words64 = r->bias_word_type == APOLLO_INDEX_I64; q.value = r->d_bias_value; q.n_bias = (int)r->n_bias;
    }
    if (r->d_mask) {
        if (r->mask_stride != 0 && r->mask_stride < (vocab + 31) / 32) return APOLLO_ERR_SHAPE;
        if ((uintptr_t)r->d_mask % 4) return APOLLO_ERR_ALIGN;
        q.mask = r->d_mask; q.mask_stride = r->mask_stride;
    }
    *out = q;
    return APOLLO_OK;
}

int check_shape(int64_t n_rows, int64_t vocab, int64_t stride, int32_t dtype)
{
    if (dtype != APOLLO_DT_F32 && dtype != APOLLO_DT_BF16) return APOLLO_ERR_INVALID_ARG;
    if (n_rows < 0 || vocab < 1 || n_rows > INT32_MAX / 8 || vocab > (int64_t)1 << 26 || stride < vocab) return APOLLO_ERR_SHAPE;
    return APOLLO_OK;
}

// How a call is cut up: chunks of the vocabulary, rows in turn.
struct Cut { int chunk, chunks, rows; };

// `most`: elements a block of threads can have of a row.  Smaller chunks while there are fewer blocks than the chip holds (a row of
// history is read once per chunk, so no smaller than that); rows that share a history in turn, as long as 16 blocks per multiprocessor remain.
Cut cut_up(int64_t n_rows, int64_t vocab, const Rules& r, int most, bool in_turn, int sms)
{
    Cut c;
    c.chunk = most;
    while (c.chunk > 1024 && n_rows * ((vocab + c.chunk - 1) / c.chunk) < 4LL * sms) c.chunk /= 2;
    c.chunks = (int)((vocab + c.chunk - 1) / c.chunk);
    int64_t rows = 1;
    if (in_turn && r.history && r.share > 1) {
        rows = n_rows * c.chunks / (16LL * sms);
        rows = rows < 1 ? 1 : rows > AJ_ROWS ? AJ_ROWS : rows;
    }
    c.rows = (int)rows;
    return c;
}

// Words of a chunk that can be listed.
int list_entries(const Rules& r, int named, int chunk)
{
    const int64_t n = (int64_t)(r.history ? r.history_len : 0) + named;
    return (int)(n < chunk ? n : chunk);
}

template <typename T>
cudaError_t run_adjust(AdjustArgs a, int sms, cudaStream_t stream)
{
    constexpr int N = Sixteen<T>::N;
    const bool place = a.logits == a.out;
    const Cut c = cut_up(a.n_rows, a.vocab, a.r, place && !a.r.bias ? AJ_PLACE_CHUNK : AJ_UNITS * AJ_THREADS * N, !(place && a.r.bias) && a.r.n_bias == 0, sms);
    a.chunk = c.chunk; a.chunks = c.chunks; a.rows = c.rows;
    a.entries = list_entries(a.r, a.r.n_bias, c.chunk);
    const int64_t blocks = (a.n_rows + c.rows - 1) / c.rows * c.chunks;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)blocks;
    if (a.r.history || a.r.n_bias) {
        const int smem = (Table::words(c.chunk, a.entries) + 2 * a.r.n_bias) * 4;
        const cudaError_t e = cudaFuncSetAttribute(adjust_kernel<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, AJ_MOST_SMEM);
        if (e != cudaSuccess) return e;
        adjust_kernel<T, true><<<grid, AJ_THREADS, smem, stream>>>(a);
    } else {
        adjust_kernel<T, false><<<grid, AJ_THREADS, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

template <typename T>
cudaError_t run_adjust_grad(AdjustGradArgs a, bool wide, int sms, int* groups, cudaStream_t stream)
{
    const int N = wide ? Sixteen<T>::N : 1;
    const bool sum = a.partial != nullptr, sparse = a.dlogits == a.dout && !sum && !a.dbias;
    Cut c;
    if (sum) {
        c.chunk = AJ_UNITS * AJ_THREADS * N;
        c.chunks = (a.vocab + c.chunk - 1) / c.chunk;
        c.rows = (int)((a.n_rows + AJ_MAX_GROUPS - 1) / AJ_MAX_GROUPS);
    } else {
        c = cut_up(a.n_rows, a.vocab, a.r, sparse ? AJ_PLACE_CHUNK : AJ_UNITS * AJ_THREADS * N, true, sms);
    }
    a.chunk = c.chunk; a.chunks = c.chunks; a.rows = c.rows;
    *groups = (int)((a.n_rows + c.rows - 1) / c.rows);
    if ((int64_t)*groups * c.chunks > INT32_MAX) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)(*groups * c.chunks);
    const int smem = a.r.history ? Table::words(c.chunk, list_entries(a.r, 0, c.chunk)) * 4 : 0;
    auto launch = [&](auto* kernel) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, AJ_MOST_SMEM);
        if (e != cudaSuccess) return e;
        kernel<<<grid, AJ_THREADS, smem, stream>>>(a);
        return cudaGetLastError();
    };
    if (!sum) return a.r.history ? launch(adjust_grad_kernel<T, true, false, true>) : launch(adjust_grad_kernel<T, false, false, true>);
    if (wide) return a.r.history ? launch(adjust_grad_kernel<T, true, true, true>) : launch(adjust_grad_kernel<T, false, true, true>);
    return a.r.history ? launch(adjust_grad_kernel<T, true, true, false>) : launch(adjust_grad_kernel<T, false, true, false>);
}

}  // namespace

}  // namespace apollo

using namespace apollo;

extern "C" int apollo_adjust_logits(const void* d_logits, int64_t row_stride, int64_t n_rows, int64_t vocab, int32_t dtype,
                                    const apollo_logit_rules* rules, void* d_out, int64_t out_stride, void* cuda_stream)
{
    int rc = check_shape(n_rows, vocab, row_stride, dtype);
    if (rc != APOLLO_OK) return rc;
    if (out_stride < vocab) return APOLLO_ERR_SHAPE;
    if (!rules) return APOLLO_ERR_INVALID_ARG;
    const size_t e = dtype == APOLLO_DT_BF16 ? 2 : 4;
    AdjustArgs a = {};
    rc = check_rules(rules, n_rows, vocab, e, false, &a.r);
    if (rc != APOLLO_OK) return rc;
    if (n_rows == 0) return APOLLO_OK;
    if (!d_logits || !d_out || (d_out == d_logits && out_stride != row_stride)) return APOLLO_ERR_INVALID_ARG;
    if ((uintptr_t)d_logits % e || (uintptr_t)d_out % e) return APOLLO_ERR_ALIGN;
    int sms = 0;
    rc = device_sms(&sms);
    if (rc != APOLLO_OK) return rc;
    a.logits = d_logits; a.out = d_out; a.stride = row_stride; a.out_stride = out_stride; a.n_rows = n_rows; a.vocab = (int)vocab;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t err = dtype == APOLLO_DT_BF16 ? run_adjust<__nv_bfloat16>(a, sms, stream) : run_adjust<float>(a, sms, stream);
    return err == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}

extern "C" int apollo_adjust_logits_grad_workspace_bytes(int64_t n_rows, int64_t vocab, size_t* out_bytes)
{
    if (!out_bytes) return APOLLO_ERR_INVALID_ARG;
    if (n_rows < 0 || vocab < 1 || n_rows > INT32_MAX / 8 || vocab > (int64_t)1 << 26) return APOLLO_ERR_SHAPE;
    *out_bytes = (size_t)(n_rows < AJ_MAX_GROUPS ? (n_rows < 1 ? 1 : n_rows) : AJ_MAX_GROUPS) * (size_t)vocab * sizeof(float);
    return APOLLO_OK;
}

extern "C" int apollo_adjust_logits_grad(const void* d_logits, int64_t row_stride, int64_t n_rows, int64_t vocab, int32_t dtype,
                                         const apollo_logit_rules* rules, const void* d_grad_out, int64_t grad_out_stride,
                                         void* d_grad_logits, int64_t grad_logits_stride, void* d_grad_bias,
                                         int64_t grad_bias_stride, float* d_grad_value, void* d_workspace,
                                         size_t workspace_bytes, void* cuda_stream)
{
    int rc = check_shape(n_rows, vocab, row_stride, dtype);
    if (rc != APOLLO_OK) return rc;
    if (grad_out_stride < vocab || grad_logits_stride < vocab || (grad_bias_stride != 0 && grad_bias_stride < vocab)) return APOLLO_ERR_SHAPE;
    if (!rules) return APOLLO_ERR_INVALID_ARG;
    const size_t e = dtype == APOLLO_DT_BF16 ? 2 : 4;
    AdjustGradArgs a = {};
    rc = check_rules(rules, n_rows, vocab, e, true, &a.r);
    if (rc != APOLLO_OK) return rc;
    const bool shared = d_grad_bias && grad_bias_stride == 0;
    if ((uintptr_t)d_logits % e || (uintptr_t)d_grad_out % e || (uintptr_t)d_grad_logits % e || (uintptr_t)d_grad_bias % e ||
        (uintptr_t)d_grad_value % 4 || (shared && (uintptr_t)d_workspace % 16))
        return APOLLO_ERR_ALIGN;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (n_rows == 0) {
        if (shared && cudaMemsetAsync(d_grad_bias, 0, (size_t)vocab * e, stream) != cudaSuccess) { cudaGetLastError(); return APOLLO_ERR_CUDA; }
        return APOLLO_OK;
    }
    if ((a.r.history && !d_logits) || !d_grad_out || !d_grad_logits || (d_grad_logits == d_grad_out && grad_logits_stride != grad_out_stride))
        return APOLLO_ERR_INVALID_ARG;
    if (shared) {
        size_t need = 0;
        rc = apollo_adjust_logits_grad_workspace_bytes(n_rows, vocab, &need);
        if (rc != APOLLO_OK) return rc;
        if (!d_workspace) return APOLLO_ERR_INVALID_ARG;
        if (workspace_bytes < need) return APOLLO_ERR_WORKSPACE;
    }
    int sms = 0;
    rc = device_sms(&sms);
    if (rc != APOLLO_OK) return rc;
    a.logits = d_logits; a.dout = d_grad_out; a.dlogits = d_grad_logits; a.dbias = shared ? nullptr : d_grad_bias;
    a.partial = shared ? static_cast<float*>(d_workspace) : nullptr; a.dvalue = a.r.n_bias ? d_grad_value : nullptr;
    a.stride = row_stride; a.dout_stride = grad_out_stride; a.dlogits_stride = grad_logits_stride; a.dbias_stride = grad_bias_stride;
    a.n_rows = n_rows; a.vocab = (int)vocab;
    // sums over rows whose vectors start at different columns go element by element
    const bool wide = !shared || whole_vectors(d_grad_logits, grad_logits_stride, e);
    int groups = 0;
    cudaError_t err = dtype == APOLLO_DT_BF16 ? run_adjust_grad<__nv_bfloat16>(a, wide, sms, &groups, stream) : run_adjust_grad<float>(a, wide, sms, &groups, stream);
    if (err == cudaSuccess && shared) {
        const unsigned grid = (unsigned)((vocab + AJ_THREADS - 1) / AJ_THREADS);
        if (dtype == APOLLO_DT_BF16) adjust_bias_join_kernel<<<grid, AJ_THREADS, 0, stream>>>(a.partial, groups, (int)vocab, static_cast<__nv_bfloat16*>(d_grad_bias));
        else adjust_bias_join_kernel<<<grid, AJ_THREADS, 0, stream>>>(a.partial, groups, (int)vocab, static_cast<float*>(d_grad_bias));
        err = cudaGetLastError();
    }
    return err == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}
