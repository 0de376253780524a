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

// What a row's table is made of, and its penalties.
struct Plan { int history, length, start; float rho, phi, pi; };

__device__ __forceinline__ Plan plan_of(const Rules& r, long long row)
{
    Plan p{ 0, 0, 0, 1.0f, 0.0f, 0.0f };
    if (r.history) {
        p.history = (int)((uint32_t)row / (uint32_t)r.share);             // (both below 2^31)
        p.length = r.length ? min(max(r.length[row], 0), r.history_len) : r.history_len;
        p.start = r.start ? min(max(r.start[row], 0), p.length) : 0;
        p.rho = r.rho_at ? r.rho_at[row] : r.rho;
        p.phi = r.phi_at ? r.phi_at[row] : r.phi;
        p.pi = r.pi_at ? r.pi_at[row] : r.pi;
    }
    return p;
}

// The table of a chunk: `chunk` words, and the list of those that are not zero.
struct Table {
    uint32_t* word;
    uint16_t* list;                      // chunk <= 65536
    int* count;
    int j0, width;
    Plan now{ -1, 0, 0, 0.0f, 0.0f, 0.0f };                // what it holds
    bool quick = false;
    int token_more, token_less;

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
        const long long first = (long long)now.history * r.history_stride;
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
    // Whether the next row's table is this one with a few tokens more, at most one a thread; then they are read now.
    __device__ __forceinline__ void look_ahead(const Rules& r, const Plan& p, int vocab)
    {
        quick = p.history == now.history && p.length >= now.length && p.length - now.length <= AJ_THREADS && p.start >= now.start &&
                p.start - now.start <= AJ_THREADS && p.start <= now.length;
        if (!quick) return;
        const long long first = (long long)p.history * r.history_stride;
        const int more = now.length + threadIdx.x, less = now.start + threadIdx.x;
        token_more = more < p.length ? token_at(r.history, first + more, r.history64, vocab) - j0 : -1;
        token_less = less < p.start ? token_at(r.history, first + less, r.history64, vocab) - j0 : -1;
    }
    // The table of a row, from that of the row before it where both have the same history.  Begins with a barrier; the caller ends with one.
    __device__ __forceinline__ void set(const Rules& r, const Plan& p, int vocab, int chunk)
    {
        auto add = [&](int j, int i) {
            if (!(atomicOr(word + j, AJ_SEEN) & AJ_SEEN)) append(j);
            if (i >= p.start) atomicAdd(word + j, 1u);
        };
        __syncthreads();
        if (quick) {
            if (token_less >= 0 && token_less < width) atomicSub(word + token_less, 1u);
            if (token_more >= 0 && token_more < width) add(token_more, now.length + (int)threadIdx.x);
        } else {
            if (p.history != now.history || p.length < now.length) {
                clear(chunk);
                __syncthreads();
                now.history = p.history;
                now.length = now.start = 0;
            }
            // positions whose count begins or ends, among those the table has
            scan(r, vocab, now.start, min(p.start, now.length), [&](int j, int) { atomicSub(word + j, 1u); });
            scan(r, vocab, p.start, min(now.start, now.length), [&](int j, int) { atomicAdd(word + j, 1u); });
            scan(r, vocab, now.length, p.length, add);
        }
        now = p;
    }
};

// Sixteen bytes of a row: N elements.  masks: a table in shared memory that makes 128-bit masks of N mask bits.
template <typename T> struct Sixteen;
template <> struct Sixteen<float> {
    static constexpr int N = 4, MASKS = 16;
    __device__ static __forceinline__ uint4 mask(int bits) { return make_uint4(-(bits & 1), -(bits >> 1 & 1), -(bits >> 2 & 1), -(bits >> 3 & 1)); }
    __device__ static __forceinline__ uint32_t minus_inf() { return 0xFF800000u; }
    __device__ static __forceinline__ void unpack(const uint4& w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    __device__ static __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
    __device__ static __forceinline__ uint4 gather(const float* p)
    {
        return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
    }
};
template <> struct Sixteen<__nv_bfloat16> {
    static constexpr int N = 8, MASKS = 256;
    __device__ static __forceinline__ uint32_t pair(int bits) { return (bits & 1) * 0xFFFFu | (bits >> 1 & 1) * 0xFFFF0000u; }
    __device__ static __forceinline__ uint4 mask(int bits) { return make_uint4(pair(bits), pair(bits >> 2), pair(bits >> 4), pair(bits >> 6)); }
    __device__ static __forceinline__ uint32_t minus_inf() { return 0xFF80FF80u; }
    __device__ static __forceinline__ void unpack(const uint4& w, float (&x)[8]) { unpack_bf16x8(w, x); }
    // (the sum of two bfloat16 rounded once)
    __device__ static __forceinline__ uint32_t add(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static __forceinline__ uint4 gather(const __nv_bfloat16* p)
    {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
        return make_uint4(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16, q[4] | (uint32_t)q[5] << 16, q[6] | (uint32_t)q[7] << 16);
    }
};

template <typename T>
__device__ __forceinline__ uint4 add16(const uint4& a, const uint4& b)
{
    return make_uint4(Sixteen<T>::add(a.x, b.x), Sixteen<T>::add(a.y, b.y), Sixteen<T>::add(a.z, b.z), Sixteen<T>::add(a.w, b.w));
}
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
// The same where j is a multiple of N: in one byte.
template <int N>
__device__ __forceinline__ uint32_t bits_in_byte(const uint32_t* words, int j)
{
    const uint32_t b = reinterpret_cast<const uint8_t*>(words)[j >> 3];
    return N == 8 ? b : b >> (j & 4) & 15u;
}
__device__ __forceinline__ bool allowed(const uint32_t* words, int j) { return !words || (words[j >> 5] >> (j & 31) & 1u); }

// A chunk of a row cut at the 16-byte boundaries of `out`: `full` vectors from column `first` on, the columns before and behind one by one.
template <typename T>
struct Span {
    static constexpr int N = Sixteen<T>::N;
    int first, full, head, tail;
    __device__ __forceinline__ Span(const T* out, int j0, int width)
    {
        head = min((int)((16u - ((uint32_t)(uintptr_t)(out + j0) & 15u)) % 16u / (uint32_t)sizeof(T)), width);
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
__device__ __forceinline__ bool on_boundary(const T* row, int first) { return ((uint32_t)(uintptr_t)(row + first) & 15u) == 0; }
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

// The logit x of a word with table entry t, before bias and mask.
__device__ __forceinline__ float penalised(float x, uint32_t t, const Plan& p)
{
    if (t & (AJ_SEEN | AJ_COUNT)) x = x > 0.0f ? __fdiv_rn(x, p.rho) : x * p.rho;
    if (t & AJ_COUNT) x -= fmaf(p.phi, (float)(t & AJ_COUNT), p.pi);
    return x;
}

// Words of a row's pairs to shared memory; a barrier later the first pair of a word sums the values of all its pairs, in order.
__device__ __forceinline__ void read_words(const Rules& r, long long row, int vocab, int* words)
{
    for (int i = threadIdx.x; i < r.n_bias; i += AJ_THREADS) words[i] = token_at(r.word, row * r.n_bias + i, r.words64, vocab);
}
__device__ __forceinline__ void sum_words(const Rules& r, long long row, Table& table, const int* words, float* sums)
{
    for (int i = threadIdx.x; i < r.n_bias; i += AJ_THREADS) {
        const int w = words[i], j = w - table.j0;
        if (w < 0 || j < 0 || j >= table.width) continue;
        bool first = true;
        for (int k = 0; k < i && first; ++k) first = words[k] != w;
        if (!first) continue;
        float sum = 0.0f;
        for (int k = i; k < r.n_bias; ++k) if (words[k] == w) sum += r.value[row * r.n_bias + k];
        sums[i] = sum;
        if (atomicOr(table.word + j, (uint32_t)(i + 1) << AJ_SLOT_SHIFT) == 0) table.append(j);
    }
}

// A row's chunk on its way through a block of threads, AJ_UNITS vectors a thread: read(), which asks for it, hold(), which puts it into shared
// memory (the columns from `held` on; up to N - 1 lie before the first boundary), each(), which takes it from there.
// EVEN: all rows start on 16-byte boundaries (and chunks are whole vectors), so addresses differ by constants.
template <typename T, bool EVEN>
struct Stream {
    using S = Sixteen<T>;
    static constexpr int N = S::N;
    uint4 ahead[AJ_UNITS];
    T ahead_single;
    T* held;
    Span<T> span;
    int single;
    __device__ __forceinline__ Stream(uint32_t* shared, const T* out, int j0, int width)
        : held(reinterpret_cast<T*>(shared) + N), span(out, j0, width), single(span.single()) {}
    static __host__ __device__ constexpr int words(int chunk) { return chunk * (int)sizeof(T) / 4 + 8; }
    __device__ __forceinline__ void place(const T* out, int j0, int width)
    {
        if constexpr (!EVEN) { span = Span<T>(out, j0, width); single = span.single(); }
    }
    __device__ __forceinline__ void read(const T* x)
    {
        if constexpr (EVEN) {
            const uint4* const p = reinterpret_cast<const uint4*>(x + span.first) + threadIdx.x;
#pragma unroll
            for (int q = 0; q < AJ_UNITS; ++q) if ((int)threadIdx.x < span.full - q * AJ_THREADS) ahead[q] = p[q * AJ_THREADS];
        } else {
            const bool aligned = on_boundary(x, span.first);
#pragma unroll
            for (int q = 0; q < AJ_UNITS; ++q) {
                const int u = q * AJ_THREADS + threadIdx.x;
                if (u < span.full) ahead[q] = load16(x + span.first + u * N, aligned);
            }
        }
        if (single >= 0) ahead_single = x[single];
    }
    __device__ __forceinline__ void hold()
    {
        uint4* const p = reinterpret_cast<uint4*>(held) + threadIdx.x;
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q) if ((int)threadIdx.x < span.full - q * AJ_THREADS) p[q * AJ_THREADS] = ahead[q];
        if (single >= 0) held[single - span.first] = ahead_single;
    }
    // out = f(vector or column, its first column), from shared memory (HELD) or as read
    template <bool HELD, typename F, typename G>
    __device__ __forceinline__ void each(T* out, F f, G g) const
    {
        const uint4* const p = reinterpret_cast<const uint4*>(held) + threadIdx.x;
        uint4* const y = reinterpret_cast<uint4*>(out + span.first) + threadIdx.x;
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q)
            if ((int)threadIdx.x < span.full - q * AJ_THREADS)
                y[q * AJ_THREADS] = f(HELD ? p[q * AJ_THREADS] : ahead[q], span.first + (q * AJ_THREADS + (int)threadIdx.x) * N, q);
        if (single >= 0) out[single] = g(HELD ? held[single - span.first] : ahead_single, single);
    }
};

// Every word of the chunk is written.  TABLE: there is a history or there are named values.  A row's logits wait in shared memory while the
// next row's are on their way; two barriers a row: one before anything reads them or the table, one between the stream's stores and those of
// the listed words.
template <typename T, bool TABLE, bool EVEN>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_kernel(const __grid_constant__ AdjustArgs a)
{
    using S = Sixteen<T>;
    constexpr int N = S::N;
    extern __shared__ __align__(16) uint32_t shared[];
    __shared__ uint4 masks[S::MASKS];
    __shared__ Plan plans[AJ_ROWS];
    __shared__ int listed;
    const int part = blockIdx.x % a.chunks;
    const long long begin = (long long)(blockIdx.x / a.chunks) * a.rows;
    const int rows = (int)min((long long)a.rows, a.n_rows - begin);
    const int j0 = part * a.chunk, width = min(a.chunk, a.vocab - j0), mask_words = (a.vocab + 31) / 32;
    const T* x0 = static_cast<const T*>(a.logits) + begin * a.stride;
    T* y0 = static_cast<T*>(a.out) + begin * a.out_stride;
    const T* b0 = a.r.bias ? static_cast<const T*>(a.r.bias) + begin * a.r.bias_stride : nullptr;
    const uint32_t* m0 = a.r.mask ? a.r.mask + begin * a.r.mask_stride : nullptr;
    Stream<T, EVEN> stream(shared, y0, j0, width);
    stream.read(x0);
    if (threadIdx.x < S::MASKS) masks[threadIdx.x] = S::mask((int)threadIdx.x);
    if (TABLE && (int)threadIdx.x < rows) plans[threadIdx.x] = plan_of(a.r, begin + threadIdx.x);
    __syncthreads();
    uint32_t* const rest = shared + Stream<T, EVEN>::words(a.chunk);
    Table table(rest, &listed, a.chunk, j0, width);
    float* const sums = reinterpret_cast<float*>(rest + Table::words(a.chunk, a.entries));
    int* const words = reinterpret_cast<int*>(sums + a.r.n_bias);
    // a vector, and a column, with bias and mask
    auto vector = [&](uint4 w, int j, int q) {
        if constexpr (EVEN) {
            if (b0) w = add16<T>(w, reinterpret_cast<const uint4*>(b0 + j0)[q * AJ_THREADS + threadIdx.x]);
            if (m0) w = select4(masks[bits_in_byte<N>(m0, j)], w, S::minus_inf());
        } else {
            if (b0) w = add16<T>(w, load16(b0 + j, on_boundary(b0, j)));
            if (m0) w = select4(masks[bits_at<N>(m0, j, mask_words)], w, S::minus_inf());
        }
        return w;
    };
    auto column = [&](T x, int j) { return !allowed(m0, j) ? (T)-INFINITY : b0 ? (T)((float)x + (float)b0[j]) : x; };
    for (int i = 0; i < rows; ++i) {
        if constexpr (!TABLE) {
            stream.template each<false>(y0, vector, column);
            if (i + 1 < rows) {
                stream.place(y0 + a.out_stride, j0, width);
                stream.read(x0 + a.stride);
            }
        } else {
            const Plan plan = plans[i];
            stream.hold();
            if (a.r.n_bias) read_words(a.r, begin + i, a.vocab, words);   // (such rows are not taken in turn)
            if (a.r.history) table.set(a.r, plan, a.vocab, a.chunk);
            else table.clear(a.chunk);
            if (a.r.n_bias) {
                __syncthreads();
                sum_words(a.r, begin + i, table, words, sums);
            }
            __syncthreads();
            const int n = listed;
            auto word = [&](int i, float& y) {         // the column of a listed word, and what it becomes
                const int k = table.list[i], j = j0 + k;
                if (!allowed(m0, j)) return -1;
                const uint32_t t = table.word[k], slot = t >> AJ_SLOT_SHIFT & AJ_SLOT;
                y = penalised((float)stream.held[j - stream.span.first], t, plan);
                if (b0) y += (float)b0[j];
                if (slot) y += sums[slot - 1];
                return j;
            };
            int at[AJ_BATCH];
            float y[AJ_BATCH];
#pragma unroll
            for (int k = 0; k < AJ_BATCH; ++k) at[k] = k * AJ_THREADS + (int)threadIdx.x < n ? word(k * AJ_THREADS + threadIdx.x, y[k]) : -1;
            if (i + 1 < rows) {
                if (a.r.history) table.look_ahead(a.r, plans[i + 1], a.vocab);
                if constexpr (EVEN) stream.read(x0 + a.stride);
            }
            stream.template each<true>(y0, vector, column);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < AJ_BATCH; ++k) if (at[k] >= 0) y0[at[k]] = (T)y[k];
            if (n > AJ_BATCH * AJ_THREADS) {
                for (int k = AJ_BATCH * AJ_THREADS + threadIdx.x; k < n; k += AJ_THREADS) {
                    const int j = word(k, y[0]);
                    if (j >= 0) y0[j] = (T)y[0];
                }
                __syncthreads();
            }
            if (!EVEN && i + 1 < rows) {
                stream.place(y0 + a.out_stride, j0, width);
                stream.read(x0 + a.stride);
            }
        }
        x0 += a.stride;
        y0 += a.out_stride;
        if (b0) b0 += a.r.bias_stride;
        if (m0) m0 += a.r.mask_stride;
    }
}

// In place without a bias: words of the history, named ones and masked ones are all that is read or written.
template <typename T>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_place_kernel(const __grid_constant__ AdjustArgs a)
{
    using S = Sixteen<T>;
    constexpr int N = S::N;
    extern __shared__ __align__(16) uint32_t shared[];
    __shared__ uint4 masks[S::MASKS];
    __shared__ int listed;
    if (threadIdx.x < S::MASKS) masks[threadIdx.x] = S::mask((int)threadIdx.x);
    const long long row = blockIdx.x / a.chunks;
    const int j0 = (int)(blockIdx.x % a.chunks) * a.chunk, width = min(a.chunk, a.vocab - j0), mask_words = (a.vocab + 31) / 32;
    Table table(shared, &listed, a.chunk, j0, width);
    float* const sums = reinterpret_cast<float*>(shared + Table::words(a.chunk, a.entries));
    int* const words = reinterpret_cast<int*>(sums + a.r.n_bias);
    T* const y0 = static_cast<T*>(a.out) + row * a.out_stride;
    const uint32_t* const m0 = a.r.mask ? a.r.mask + row * a.r.mask_stride : nullptr;
    const Plan p = plan_of(a.r, row);
    if (a.r.n_bias) read_words(a.r, row, a.vocab, words);
    if (a.r.history) table.set(a.r, p, a.vocab, a.chunk);
    else table.clear(a.chunk);
    if (a.r.n_bias) {
        __syncthreads();
        sum_words(a.r, row, table, words, sums);
    }
    __syncthreads();
    const int n = listed;
    for (int i = threadIdx.x; i < n; i += AJ_THREADS * AJ_BATCH) {
        int at[AJ_BATCH];
        T x[AJ_BATCH];
#pragma unroll
        for (int k = 0; k < AJ_BATCH; ++k) {
            at[k] = i + k * AJ_THREADS < n ? table.list[i + k * AJ_THREADS] : -1;
            if (at[k] >= 0 && !allowed(m0, j0 + at[k])) at[k] = -1;
            if (at[k] >= 0) x[k] = y0[j0 + at[k]];
        }
#pragma unroll
        for (int k = 0; k < AJ_BATCH; ++k) {
            if (at[k] < 0) continue;
            const uint32_t t = table.word[at[k]], slot = t >> AJ_SLOT_SHIFT & AJ_SLOT;
            const float y = penalised((float)x[k], t, p);
            y0[j0 + at[k]] = (T)(slot ? y + sums[slot - 1] : y);
        }
    }
    if (!m0) return;
    __syncthreads();                                   // a vector with a masked word may hold one of those
    const Span<T> span(y0, j0, width);
    for (int u = threadIdx.x; u < span.full; u += AJ_THREADS) {
        const int j = span.first + u * N;
        const uint32_t live = bits_at<N>(m0, j, mask_words);
        if (live == (1u << N) - 1u) continue;
        uint4* const y = reinterpret_cast<uint4*>(y0 + j);
        *y = select4(masks[live], live ? *y : make_uint4(0, 0, 0, 0), S::minus_inf());
    }
    if (const int j = span.single(); j >= 0 && !allowed(m0, j)) y0[j] = (T)-INFINITY;
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
    __shared__ uint4 masks[S::MASKS];
    __shared__ int listed;
    if (threadIdx.x < S::MASKS) masks[threadIdx.x] = S::mask((int)threadIdx.x);
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
    Plan plan{};
    if constexpr (TABLE) plan = plan_of(a.r, begin);
    for (long long row = begin; row < end; ++row) {
        Plan next{};
        if (TABLE && row + 1 < end) next = plan_of(a.r, row + 1);
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
            rho = plan.rho;
            table.set(a.r, plan, a.vocab, a.chunk);
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
                    if (m0) w = select4(masks[span.first % N == 0 ? bits_in_byte<N>(m0, j) : bits_at<N>(m0, j, mask_words)], w, 0);
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
                    *y = select4(masks[live], live ? *y : make_uint4(0, 0, 0, 0), 0);
                }
            }
            if (const int j = span.single(); j >= 0) column(j, edge);
        }
        if constexpr (TABLE) {
            if (row + 1 < end) table.look_ahead(a.r, next, a.vocab);
            plan = next;
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
        q.length = r->d_length; q.start = gradient ? nullptr : r->d_start;
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
    const bool sparse = a.logits == a.out && !a.r.bias;
    const Cut c = cut_up(a.n_rows, a.vocab, a.r, sparse ? AJ_PLACE_CHUNK : AJ_UNITS * AJ_THREADS * N, !sparse && a.r.n_bias == 0, sms);
    a.chunk = c.chunk; a.chunks = c.chunks; a.rows = c.rows;
    a.entries = list_entries(a.r, a.r.n_bias, c.chunk);
    const int64_t blocks = (a.n_rows + c.rows - 1) / c.rows * c.chunks;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    const bool table = a.r.history || a.r.n_bias;
    if (sparse && !table && !a.r.mask) return cudaSuccess;
    const int smem = sparse ? (Table::words(c.chunk, a.entries) + 2 * a.r.n_bias) * 4
                            : table ? (Table::words(c.chunk, a.entries) + 2 * a.r.n_bias + Stream<T, true>::words(c.chunk)) * 4 : 0;
    auto launch = [&](auto* kernel) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, AJ_MOST_SMEM);
        if (e != cudaSuccess) return e;
        kernel<<<(unsigned)blocks, AJ_THREADS, smem, stream>>>(a);
        return cudaGetLastError();
    };
    if (sparse) return launch(adjust_place_kernel<T>);
    const bool even = whole_vectors(a.logits, a.stride, sizeof(T)) && whole_vectors(a.out, a.out_stride, sizeof(T)) && whole_vectors(a.r.bias, a.r.bias_stride, sizeof(T));
    if (table) return even ? launch(adjust_kernel<T, true, true>) : launch(adjust_kernel<T, true, false>);
    return even ? launch(adjust_kernel<T, false, true>) : launch(adjust_kernel<T, false, false>);
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
