// Logits adjusted by penalties for repeated tokens, biases and grammar masks, and the gradient of that.
//
//   c_j, d_j = occurrences of word j in the row's history, and from position `start` on
//   x = logit_j;  c_j > 0: x <- x > 0 ? x / rho : x rho;  d_j > 0: x <- x - (phi d_j + pi);  x <- x + bias_j + named values;
//   mask bit 0: x <- -inf
//   a_j = allowed ? dout_j : 0;  dlogit_j = a_j {1, 1 / rho, rho};  dbias_j = a_j (summed over rows if shared);  dvalue_i = a_j
//
// Two kernels.  One streams over rows and knows of bias and mask alone.  The other takes a chunk of the vocabulary for one row, or for a few
// rows in turn: it counts the tokens of its chunk in a table in shared memory and lists the words that occur (integer atomics: their
// order decides the order of the list, not the results), then writes the listed words, one a thread.  In place the second one
// does everything: without a bias the listed words and the masked ones are all that changes.  Rows that share a history (the positions of a sequence in
// training) go on with the table of the row before: they add the tokens in between.  A table word holds
// [31] seen at all  [30..20] 1 + slot of the word's named value  [19..0] how often from `start` on;  of short histories half of that.
// What was tried: vectors that look into the table (in a training batch nearly every warp had a word to look up: 376 instructions a
// vector of eight; 8192 x 32000 bfloat16 785 us), both passes in one kernel with barriers between them (351 us), the same with the next row's
// loads under way (266 us, at three times the code), the words of some rows beside the stream of the next ones in one launch (six slabs of rows:
// 375 us, the blocks of words are the long ones).
// 8192 x 32000 bfloat16 with a bias and a mask: stream 153 us, 6.9 TB/s (its sums over rows for a bias' gradient: 170 us, 6.2 TB/s; rows ahead in
// shared memory made that no faster: 296 instead of 292 us for the whole gradient); words of histories of 512 tokens on average, 2 M of them: 97 us
// (113 with 32-bit entries), gradient 103 us, where warps wait for barriers (5 cycles an instruction) and memory is at 16 %.
#include "../../include/apollo.h"

#include <cmath>

#include "device_utils.cuh"
#include "host_utils.h"
#include "tc_ptx.cuh"

namespace apollo {

namespace {

constexpr int AJ_THREADS = 256;
constexpr int AJ_UNITS = 4;              // vectors a thread has of a row's chunk at once
constexpr int AJ_STEP = 8;               // rows whose strides make a multiple of 16 bytes
// Rows of partial sums for a shared bias, a multiple of AJ_STEP (8192 x 32000: 128 284 us, 256 290).
constexpr int AJ_MAX_GROUPS = 128;
constexpr int AJ_ROWS = 16;              // most rows in turn
constexpr int AJ_SHORT = 4096;           // tokens of a history that is counted in 16 bits (at most 2^15 - 1)
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

// A token, or -1 for one outside [0, vocab) (whatever it is: the caller subtracts the first word of a chunk from it).
__device__ __forceinline__ int token_at(const void* p, long long i, int is64, int vocab)
{
    if (is64) {
        const unsigned long long v = static_cast<const unsigned long long*>(p)[i];
        return v < (unsigned long long)vocab ? (int)v : -1;
    }
    const unsigned v = static_cast<const unsigned*>(p)[i];
    return v < (unsigned)vocab ? (int)v : -1;
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

__host__ __device__ constexpr int four(int n) { return (n + 3) / 4 * 4; }

// The table of a chunk: `chunk` entries, and the list of those that are not zero.  HALF: entries of 16 bits, two in a word ([15] seen at all
// [14..0] how often): histories of up to AJ_SHORT tokens, no named values.  Half the shared memory, so twice the blocks, of half the threads.
template <bool HALF>
struct Table {
    static constexpr int THREADS = HALF ? AJ_THREADS / 2 : AJ_THREADS;
    // Scattered loads that a thread has in flight.  Long histories: 8, 21.8 us for 129 rows of 8191 tokens (4: 26.3, 16: 29.3 and 36.8).  Short ones,
    // most of them a few tokens more than the row before: 4 (8: 8192 x 32000 261 us for 254).
    static constexpr int BATCH = HALF ? 4 : 8;
    uint32_t* word;
    uint16_t* list;                      // chunk <= 65536
    int* count;
    int j0, width;
    Plan now{ -1, 0, 0, 0.0f, 0.0f, 0.0f };                // what it holds
    bool quick = false;
    int token_more, token_less;

    __device__ __forceinline__ Table(uint32_t* at, int* n, int chunk, int first, int w)
        : word(at), list(reinterpret_cast<uint16_t*>(at + (HALF ? chunk / 2 : chunk))), count(n), j0(first), width(w) {}
    static __host__ __device__ constexpr int words(int chunk, int entries) { return (HALF ? chunk / 2 : chunk) + (entries + 1) / 2; }
    __device__ __forceinline__ void clear(int chunk)
    {
        for (int i = threadIdx.x * 4; i < (HALF ? chunk / 2 : chunk); i += THREADS * 4) *reinterpret_cast<uint4*>(word + i) = make_uint4(0, 0, 0, 0);
        if (threadIdx.x == 0) *count = 0;
    }
    // An entry as [31] seen [30..20] slot [19..0] how often.
    __device__ __forceinline__ uint32_t entry(int j) const
    {
        if constexpr (!HALF) return word[j];
        const uint32_t e = word[j >> 1] >> (16 * (j & 1));
        return (e & 0x8000u) << 16 | (e & 0x7FFFu);
    }
    // Whether the word has been seen before; from now on it has, and with `counted` once more.
    __device__ __forceinline__ bool see(int j, bool counted)
    {
        if constexpr (!HALF) {
            const bool before = atomicOr(word + j, AJ_SEEN) & AJ_SEEN;
            if (counted) atomicAdd(word + j, 1u);
            return before;
        }
        const int shift = 16 * (j & 1);
        const bool before = atomicOr(word + (j >> 1), 0x8000u << shift) >> shift & 0x8000u;
        if (counted) atomicAdd(word + (j >> 1), 1u << shift);
        return before;
    }
    __device__ __forceinline__ void count_more(int j)
    {
        if constexpr (HALF) atomicAdd(word + (j >> 1), 1u << (16 * (j & 1)));
        else atomicAdd(word + j, 1u);
    }
    __device__ __forceinline__ void count_less(int j)
    {
        if constexpr (HALF) atomicSub(word + (j >> 1), 1u << (16 * (j & 1)));
        else atomicSub(word + j, 1u);
    }
    __device__ __forceinline__ void append(int j) { list[atomicAdd(count, 1)] = (uint16_t)j; }
    // f(word, position) for the tokens of the chunk at positions [from, to).
    template <typename F>
    __device__ __forceinline__ void scan(const Rules& r, int vocab, int from, int to, F f)
    {
        const long long first = (long long)now.history * r.history_stride;
        for (int i = from + (int)threadIdx.x; i < to; i += THREADS * BATCH) {
            int j[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int at = i + k * THREADS;
                j[k] = at < to ? token_at(r.history, first + at, r.history64, vocab) - j0 : -1;
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) if (j[k] >= 0 && j[k] < width) f(j[k], i + k * THREADS);
        }
    }
    // Whether the next row's table is this one with a few tokens more, at most one a thread; then they are read now.
    __device__ __forceinline__ void look_ahead(const Rules& r, const Plan& p, int vocab)
    {
        quick = p.history == now.history && p.length >= now.length && p.length - now.length <= THREADS && p.start >= now.start &&
                p.start - now.start <= THREADS && p.start <= now.length;
        if (!quick) return;
        const long long first = (long long)p.history * r.history_stride;
        const int more = now.length + threadIdx.x, less = now.start + threadIdx.x;
        token_more = more < p.length ? token_at(r.history, first + more, r.history64, vocab) - j0 : -1;
        token_less = less < p.start ? token_at(r.history, first + less, r.history64, vocab) - j0 : -1;
    }
    // The table of a row, from that of the row before it where both have the same history.  Between two barriers of the caller's.
    __device__ __forceinline__ void set(const Rules& r, const Plan& p, int vocab, int chunk)
    {
        auto add = [&](int j, int i) {
            if (!see(j, i >= p.start)) append(j);
        };
        if (quick) {
            if (token_less >= 0 && token_less < width) count_less(token_less);
            if (token_more >= 0 && token_more < width) add(token_more, now.length + (int)threadIdx.x);
        } else {
            if (p.history != now.history || p.length < now.length) {
                clear(chunk);
                __syncthreads();
                now.history = p.history;
                now.length = now.start = 0;
            }
            // positions whose count begins or ends, among those the table has
            scan(r, vocab, now.start, min(p.start, now.length), [&](int j, int) { count_less(j); });
            scan(r, vocab, p.start, min(now.start, now.length), [&](int j, int) { count_more(j); });
            scan(r, vocab, now.length, p.length, add);
        }
        now = p;
    }
};

// Sixteen bytes of a row: N elements.  Entry: of the table in shared memory that makes element masks of four mask bits.
template <typename T> struct Sixteen;
template <> struct Sixteen<float> {
    static constexpr int N = 4;
    using Entry = uint4;
    __device__ static __forceinline__ Entry entry(int bits) { return make_uint4(-(bits & 1), -(bits >> 1 & 1), -(bits >> 2 & 1), -(bits >> 3 & 1)); }
    __device__ static __forceinline__ uint4 masks(const Entry* t, uint32_t bits) { return t[bits]; }
    static constexpr uint32_t MINUS_INF = 0xFF800000u;
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
    static constexpr int N = 8;
    using Entry = uint2;
    __device__ static __forceinline__ uint32_t pair(int bits) { return (bits & 1) * 0xFFFFu | (bits >> 1 & 1) * 0xFFFF0000u; }
    __device__ static __forceinline__ Entry entry(int bits) { return make_uint2(pair(bits), pair(bits >> 2)); }
    __device__ static __forceinline__ uint4 masks(const Entry* t, uint32_t bits)
    {
        const uint2 a = t[bits & 15], b = t[bits >> 4];
        return make_uint4(a.x, a.y, b.x, b.y);
    }
    static constexpr uint32_t MINUS_INF = 0xFF80FF80u;
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
        // (words of 32 bits from the first boundary on: a bias shared by odd rows, 4096 x 50257, 135 us; eight halves each 170)
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
        const int odd = (uint32_t)(uintptr_t)p >> 1 & 1;
        const uint32_t* const w = reinterpret_cast<const uint32_t*>(q + odd);
        if (!odd) return make_uint4(w[0], w[1], w[2], w[3]);
        const uint32_t first = q[0], last = q[7];
        return make_uint4(first | w[0] << 16, __funnelshift_r(w[0], w[1], 16), __funnelshift_r(w[1], w[2], 16), w[2] >> 16 | last << 16);
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
    const uint32_t lo = __ldg(words + w), hi = at + N > 32 && w + 1 < n_words ? __ldg(words + w + 1) : 0;
    return __funnelshift_r(lo, hi, at) & ((1u << N) - 1u);
}
// The same where j is a multiple of N: in one byte.
template <int N>
__device__ __forceinline__ uint32_t bits_in_byte(const uint32_t* words, int j)
{
    const uint32_t b = __ldg(reinterpret_cast<const uint8_t*>(words) + (j >> 3));
    return N == 8 ? b : b >> (j & 4) & 15u;
}
__device__ __forceinline__ bool allowed(const uint32_t* words, int j) { return !words || (__ldg(words + (j >> 5)) >> (j & 31) & 1u); }

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

// The logit x of a word with table entry t, before bias and mask.
__device__ __forceinline__ float penalised(float x, uint32_t t, const Plan& p)
{
    if (t & (AJ_SEEN | AJ_COUNT)) x = x > 0.0f ? __fdiv_rn(x, p.rho) : x * p.rho;
    if (t & AJ_COUNT) x -= fmaf(p.phi, (float)(t & AJ_COUNT), p.pi);
    return x;
}

// Words of a row's pairs to shared memory (-1 up to a multiple of four); a barrier later the first pair of a word sums the values of all its
// pairs, in order.  Four words a look, no look depends on the one before it; only a word that is named again is looked for once more.
template <int THREADS>
__device__ __forceinline__ void read_words(const Rules& r, long long row, int vocab, int* words)
{
    for (int i = threadIdx.x; i < four(r.n_bias); i += THREADS) words[i] = i < r.n_bias ? token_at(r.word, row * r.n_bias + i, r.words64, vocab) : -1;
}
template <int THREADS>
__device__ __forceinline__ void sum_words(const Rules& r, long long row, Table<false>& table, const int* words, float* sums)
{
    for (int i = threadIdx.x; i < r.n_bias; i += THREADS) {
        const int w = words[i], j = w - table.j0;
        if (w < 0 || j < 0 || j >= table.width) continue;
        const float* const values = r.value + row * r.n_bias;
        float sum = values[i];
        int earlier = 0, all = 0;
#pragma unroll 4
        for (int k = 0; k < r.n_bias; k += 4) {
            const int4 q = *reinterpret_cast<const int4*>(words + k);
            const int same[4] = { q.x == w, q.y == w, q.z == w, q.w == w };
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                all += same[x];
                earlier += same[x] && k + x < i;
            }
        }
        if (earlier) continue;
        if (all > 1)
            for (int k = i + 1; k < r.n_bias; ++k) if (words[k] == w) sum += values[k];
        sums[i] = sum;
        if (atomicOr(table.word + j, (uint32_t)(i + 1) << AJ_SLOT_SHIFT) == 0) table.append(j);
    }
}

// What a vector, or a column, becomes on the way: bias, mask.  OTHER: what a masked word becomes.
template <typename T>
struct Dense {
    using S = Sixteen<T>;
    static constexpr int N = S::N;
    const T* bias;
    const uint32_t* mask;
    const typename S::Entry* masks;
    uint32_t other;
    int mask_words;
    template <bool EVEN>
    __device__ __forceinline__ uint4 vector(uint4 w, int j) const
    {
        if (bias) w = add16<T>(w, EVEN ? __ldg(reinterpret_cast<const uint4*>(bias + j)) : load16(bias + j, on_boundary(bias, j)));
        if (mask) w = select4(S::masks(masks, EVEN ? bits_in_byte<N>(mask, j) : bits_at<N>(mask, j, mask_words)), w, other);
        return w;
    }
    __device__ __forceinline__ T column(T x, int j) const
    {
        return !allowed(mask, j) ? (other ? (T)-INFINITY : (T)0.0f) : bias ? (T)((float)x + (float)bias[j]) : x;
    }
};

struct StreamArgs {
    const void* in;
    void* out;                           // may be `in`
    void* copy;                          // the same once more (rows of a bias), or null
    float* partial;                      // SUM: sums over the rows of a block of threads, vocab floats each
    const void* bias;
    const uint32_t* mask;
    long long in_stride, out_stride, copy_stride, bias_stride, mask_stride, n_rows;
    uint32_t other;
    int vocab, chunk, chunks, rows;      // rows: of a block of threads (1 unless they are summed), every AJ_STEP-th
};

// Four vectors a thread, all loads before the first store.  EVEN: all rows start on 16-byte boundaries, so addresses differ by constants.
// SUM: the sums over a block's rows stay in registers.  Every row's vectors have to start at the same columns then: a block has every eighth
// row, which start alike whatever the stride (4096 x 50257 bfloat16 225 us; rows in order, column by column: 406), and the sums' order does
// not depend on the layout.
template <typename T, bool EVEN, bool SUM>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_stream_kernel(const __grid_constant__ StreamArgs a)
{
    using S = Sixteen<T>;
    constexpr int N = S::N;
    __shared__ typename S::Entry masks[16];
    ptx::grid_launch_dependents();
    if (threadIdx.x < 16) masks[threadIdx.x] = S::entry((int)threadIdx.x);
    __syncthreads();
    const int tid = threadIdx.x, part = blockIdx.x % a.chunks;
    const long long group = blockIdx.x / a.chunks, step = SUM ? AJ_STEP : 1, begin = SUM ? group % step + group / step * step * a.rows : group;
    const int rows = SUM ? (int)max(0ll, min((long long)a.rows, (a.n_rows - begin + step - 1) / step)) : 1;
    const int j0 = part * a.chunk, width = min(a.chunk, a.vocab - j0);
    const T* x0 = static_cast<const T*>(a.in) + begin * a.in_stride;
    T* y0 = static_cast<T*>(a.out) + begin * a.out_stride;
    T* c0 = a.copy ? static_cast<T*>(a.copy) + begin * a.copy_stride : nullptr;
    Dense<T> dense{ a.bias ? static_cast<const T*>(a.bias) + begin * a.bias_stride : nullptr, a.mask ? a.mask + begin * a.mask_stride : nullptr,
                    masks, a.other, (a.vocab + 31) / 32 };
    const bool keep = a.in == a.out && !a.bias && !a.mask;                // nothing to write there
    float sum[SUM ? AJ_UNITS : 1][N], edge = 0.0f;
#pragma unroll
    for (int q = 0; q < (SUM ? AJ_UNITS : 1); ++q)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[q][e] = 0.0f;
    const Span<T> span(y0, j0, width);
    for (int i = 0; i < rows; ++i) {
        const bool aligned = EVEN || on_boundary(x0, span.first), c_aligned = EVEN || (c0 && on_boundary(c0, span.first)), plain = span.first % N == 0;
        uint4 w[AJ_UNITS];
        const T* const x = x0 + span.first + tid * N;
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q) if (tid < span.full - q * AJ_THREADS) w[q] = load16(x + q * AJ_THREADS * N, aligned);
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q) {
            if (tid >= span.full - q * AJ_THREADS) continue;
            const int j = span.first + (q * AJ_THREADS + tid) * N;
            w[q] = EVEN || (plain && !dense.bias) ? dense.template vector<true>(w[q], j) : dense.template vector<false>(w[q], j);
            if constexpr (SUM) {
                float g[N];
                S::unpack(w[q], g);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[q][e] += g[e];
            }
        }
        T* const y = y0 + span.first + tid * N;
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q) {
            if (tid >= span.full - q * AJ_THREADS) continue;
            if (!keep) *reinterpret_cast<uint4*>(y + q * AJ_THREADS * N) = w[q];
            if (c0) {
                T* const c = c0 + span.first + (q * AJ_THREADS + tid) * N;
                if (c_aligned) {
                    *reinterpret_cast<uint4*>(c) = w[q];
                } else {
                    float g[N];
                    S::unpack(w[q], g);
#pragma unroll
                    for (int e = 0; e < N; ++e) c[e] = (T)g[e];
                }
            }
        }
        if (const int j = span.single(); j >= 0) {
            const T r = dense.column(x0[j], j);
            y0[j] = r;
            if (c0) c0[j] = r;
            if constexpr (SUM) edge += (float)r;
        }
        x0 += step * a.in_stride;
        y0 += step * a.out_stride;
        if (c0) c0 += a.copy_stride;
        if (dense.bias) dense.bias += a.bias_stride;
        if (dense.mask) dense.mask += step * a.mask_stride;
    }
    if constexpr (SUM) {
        float* const p = a.partial + group * a.vocab;
#pragma unroll
        for (int q = 0; q < AJ_UNITS; ++q) {
            if (tid >= span.full - q * AJ_THREADS) continue;
#pragma unroll
            for (int e = 0; e < N; ++e) p[span.first + (q * AJ_THREADS + tid) * N + e] = sum[q][e];
        }
        if (const int j = span.single(); j >= 0) p[j] = edge;
    }
}

// What the kernel of the listed words does beside them.
enum : int {
    AJ_WORDS_ONLY = 0,                   // the stream has written the others
    AJ_MASKED_TOO = 1,                   // in place: the masked words
    AJ_ALL_TOO = 2,                      // in place with a bias: every other word (one row a block; the listed words' results wait in the table, the
                                         // row is on its way while the table is made)
};

struct WordsArgs {
    const void* logits;
    const void* dout;                    // gradient: of the adjusted logits
    void* out;                           // adjusted logits, or the gradient of the logits
    float* dvalue;
    long long stride, dout_stride, out_stride, n_rows;
    uint32_t other;
    int vocab, chunk, chunks, rows;      // rows: in turn
    int entries;                         // of the list at most
    int mode;
    Rules r;
};

// Blocks a multiprocessor that the registers are to allow: it decides how the compiler orders the scattered loads.  Short histories, forward:
// 12 (8192 x 32000 bfloat16 257 us, 4096 x 50256 in place 57.5; 6 255 and 65.7; 9 260 and 59.5); gradient: bfloat16 6 (8192 x 32000 304 us,
// 9 330), fp32 9 (777 x 50001 88 us, 6 90; why the types differ is not known, the bounds are what these shapes took).  Others 4: what shared memory holds (in place with a bias, 4096 x 50256 bfloat16: 280 us, 5 344).
constexpr int words_resident(bool half, bool grad, size_t e) { return !half ? 4 : !grad ? 12 : e == 2 ? 6 : 9; }

// ALL: mode AJ_ALL_TOO.
template <typename T, bool GRAD, bool HALF, bool ALL>
__global__ void __launch_bounds__(Table<HALF>::THREADS, words_resident(HALF, GRAD, sizeof(T)))
adjust_words_kernel(const __grid_constant__ WordsArgs a)
{
    using S = Sixteen<T>;
    constexpr int N = S::N, THREADS = Table<HALF>::THREADS;
    extern __shared__ __align__(16) uint32_t shared[];
    __shared__ typename S::Entry masks[16];
    __shared__ Plan plans[AJ_ROWS];
    __shared__ int listed;
    // (the first chunk's blocks first: where common words have low numbers they are the long ones)
    const unsigned groups = gridDim.x / (unsigned)a.chunks;
    const int part = (int)(blockIdx.x / groups);
    const long long begin = (long long)(blockIdx.x % groups) * a.rows;
    const int rows = (int)min((long long)a.rows, a.n_rows - begin);
    const int j0 = part * a.chunk, width = min(a.chunk, a.vocab - j0);
    if (threadIdx.x < 16) masks[threadIdx.x] = S::entry((int)threadIdx.x);
    if ((int)threadIdx.x < rows) plans[threadIdx.x] = plan_of(a.r, begin + threadIdx.x);
    Table<HALF> table(shared, &listed, a.chunk, j0, width);
    int* const words = reinterpret_cast<int*>(shared + four(Table<HALF>::words(a.chunk, a.entries)));
    float* const sums = reinterpret_cast<float*>(words + (GRAD ? 0 : four(a.r.n_bias)));
    table.clear(a.chunk);
    __syncthreads();
    table.now.history = plans[0].history;              // with nothing of it yet
    bool waited = a.mode != AJ_WORDS_ONLY;             // for the stream: its stores come first
    for (int i = 0; i < rows; ++i) {
        const long long row = begin + i;
        const Plan plan = plans[i];
        const T* const x0 = static_cast<const T*>(a.logits) + row * a.stride;
        const T* const g0 = GRAD ? static_cast<const T*>(a.dout) + row * a.dout_stride : nullptr;
        T* const y0 = static_cast<T*>(a.out) + row * a.out_stride;
        const T* const b0 = !GRAD && a.r.bias ? static_cast<const T*>(a.r.bias) + row * a.r.bias_stride : nullptr;
        const uint32_t* const m0 = a.r.mask ? a.r.mask + row * a.r.mask_stride : nullptr;
        const Span<T> span(y0, j0, width);
        uint4 w[AJ_UNITS];
        auto load = [&](int first) {
#pragma unroll
            for (int q = 0; q < AJ_UNITS; ++q)
                if (const int u = first + q * THREADS; u < span.full) w[q] = *reinterpret_cast<const uint4*>(y0 + span.first + u * N);
        };
        if constexpr (ALL) load(threadIdx.x);
        if constexpr (!GRAD && !HALF) if (a.r.n_bias) read_words<THREADS>(a.r, row, a.vocab, words);       // (such rows are not taken in turn)
        if (a.r.history) table.set(a.r, plan, a.vocab, a.chunk);
        if constexpr (GRAD) {
            // (in place: before anything of the row is overwritten)
            if (a.dvalue)
                for (int k = threadIdx.x; k < a.r.n_bias; k += THREADS) {
                    const int w = token_at(a.r.word, row * a.r.n_bias + k, a.r.words64, a.vocab);
                    if (w < 0 ? j0 == 0 : w >= j0 && w < j0 + width) a.dvalue[row * a.r.n_bias + k] = w >= 0 && allowed(m0, w) ? (float)g0[w] : 0.0f;
                }
        } else if constexpr (!HALF) {
            if (a.r.n_bias) {
                __syncthreads();
                sum_words<THREADS>(a.r, row, table, words, sums);
            }
        }
        __syncthreads();
        const int n = listed;
        if (i + 1 < rows && a.r.history) table.look_ahead(a.r, plans[i + 1], a.vocab);
        // what a listed word becomes
        auto result = [&](int k, float x, float g) {
            const uint32_t t = table.entry(k);
            if constexpr (GRAD) return x > 0.0f ? __fdiv_rn(g, plan.rho) : g * plan.rho;
            float y = penalised(x, t, plan);
            if (b0) y += (float)b0[j0 + k];
            const uint32_t slot = t >> AJ_SLOT_SHIFT & AJ_SLOT;
            return slot ? y + sums[slot - 1] : y;
        };
        for (int first = threadIdx.x; first < n; first += THREADS * Table<HALF>::BATCH) {
            int at[Table<HALF>::BATCH];
            T x[Table<HALF>::BATCH], g[Table<HALF>::BATCH];
#pragma unroll
            for (int k = 0; k < Table<HALF>::BATCH; ++k) {
                at[k] = first + k * THREADS < n ? table.list[first + k * THREADS] : -1;
                if (at[k] >= 0 && !allowed(m0, j0 + at[k])) at[k] = -1;
                if (at[k] >= 0) {
                    x[k] = x0[j0 + at[k]];
                    if constexpr (GRAD) g[k] = g0[j0 + at[k]];
                }
            }
            if (!waited) { ptx::grid_wait_previous(); waited = true; }
#pragma unroll
            for (int k = 0; k < Table<HALF>::BATCH; ++k) {
                if (at[k] < 0) continue;
                const float y = result(at[k], (float)x[k], GRAD ? (float)g[k] : 0.0f);
                if constexpr (ALL) table.word[at[k]] = __float_as_uint(y);
                else y0[j0 + at[k]] = (T)y;
            }
        }
        __syncthreads();                               // done with the table, and with vectors that hold listed words and masked ones
        if (!ALL && (a.mode == AJ_WORDS_ONLY || !m0)) continue;
        const Dense<T> dense{ b0, m0, masks, a.other, (a.vocab + 31) / 32 };
        auto at = [&](int u) { return reinterpret_cast<uint4*>(y0 + span.first + u * N); };
        if constexpr (ALL) {
            for (int first = threadIdx.x; first < span.full; first += THREADS * AJ_UNITS) {
                if (first != (int)threadIdx.x) load(first);
#pragma unroll
                for (int q = 0; q < AJ_UNITS; ++q)
                    if (const int u = first + q * THREADS; u < span.full) *at(u) = dense.template vector<false>(w[q], span.first + u * N);
            }
        } else {
            for (int u = threadIdx.x; u < span.full; u += THREADS) {
                const uint32_t live = bits_at<N>(m0, span.first + u * N, dense.mask_words);
                if (live != (1u << N) - 1u) *at(u) = select4(S::masks(masks, live), live ? *at(u) : make_uint4(0, 0, 0, 0), a.other);
            }
        }
        if (const int j = span.single(); j >= 0 && (ALL || !allowed(m0, j))) y0[j] = dense.column(y0[j], j);
        if constexpr (ALL) {
            __syncthreads();
            for (int k = threadIdx.x; k < n; k += THREADS) {
                const int j = table.list[k];
                if (allowed(m0, j0 + j)) y0[j0 + j] = (T)__uint_as_float(table.word[j]);
            }
        }
    }
    if (!waited) ptx::grid_wait_previous();            // what comes next in the stream may count on both
}

// Sums over the groups of rows: a warp takes every eighth group for 32 columns, the eight sums are added in order (256 groups of 32000: 8 us, 20 us with
// one thread for all groups of a column).
template <typename T>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_bias_join_kernel(const float* __restrict__ partial, int groups, int vocab, T* __restrict__ dbias)
{
    constexpr int WARPS = AJ_THREADS / 32;
    __shared__ float sums[WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (j < vocab) {
#pragma unroll 8
        for (int g = warp; g < groups; g += WARPS) sum += partial[(long long)g * vocab + j];
    }
    sums[warp][lane] = sum;
    __syncthreads();
    if (warp > 0 || j >= vocab) return;
#pragma unroll
    for (int w = 1; w < WARPS; ++w) sum += sums[w][lane];
    dbias[j] = (T)sum;
}

constexpr int AJ_WORDS_CHUNK = 8192;
constexpr int AJ_DEPTH = 64;
constexpr int AJ_MOST_SMEM = (four(Table<false>::words(AJ_WORDS_CHUNK, AJ_WORDS_CHUNK)) + 2 * APOLLO_MAX_BIAS_WORDS) * 4;

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

// Words of a chunk that can be listed.
int list_entries(const Rules& r, int named, int chunk)
{
    const int64_t n = (int64_t)(r.history ? r.history_len : 0) + named;
    return (int)(n < chunk ? n : chunk);
}

// Launches the stream.  Small calls in smaller chunks, so that every multiprocessor has a block.
template <typename T>
cudaError_t run_stream(StreamArgs a, int sms, int* groups, cudaStream_t stream)
{
    constexpr size_t e = sizeof(T);
    const bool sum = a.partial != nullptr;
    const bool even = whole_vectors(a.in, a.in_stride, e) && whole_vectors(a.out, a.out_stride, e) && whole_vectors(a.copy, a.copy ? a.copy_stride : 0, e) &&
                      whole_vectors(a.bias, a.bias ? a.bias_stride : 0, e);
    a.chunk = AJ_UNITS * AJ_THREADS * Sixteen<T>::N;
    if (!sum)
        while (a.chunk > 2048 && a.n_rows * ((a.vocab + a.chunk - 1) / a.chunk) < 2LL * sms) a.chunk /= 2;
    a.chunks = (a.vocab + a.chunk - 1) / a.chunk;
    a.rows = 1;
    int64_t n = a.n_rows;
    if (sum) {
        const int64_t each = (a.n_rows + AJ_STEP - 1) / AJ_STEP, most = AJ_MAX_GROUPS / AJ_STEP;
        a.rows = (int)((each + most - 1) / most);
        if (a.rows > 1) n = (each + a.rows - 1) / a.rows * AJ_STEP;       // (one row each: group and row have the same number)
    }
    *groups = (int)n;
    if (n * a.chunks > INT32_MAX) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)(n * a.chunks);
    if (sum) {
        if (even) adjust_stream_kernel<T, true, true><<<grid, AJ_THREADS, 0, stream>>>(a);
        else adjust_stream_kernel<T, false, true><<<grid, AJ_THREADS, 0, stream>>>(a);
    } else {
        if (even) adjust_stream_kernel<T, true, false><<<grid, AJ_THREADS, 0, stream>>>(a);
        else adjust_stream_kernel<T, false, false><<<grid, AJ_THREADS, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

// Launches the kernel of the listed words, after the stream where that has run (only then may its blocks start early: what else comes before
// it in the caller's stream may write what it reads).  Chunks as large as shared memory holds for several blocks
// (a row of the history is read once per chunk), smaller ones while there are fewer blocks than the chip holds; rows that share a history in
// turn, as long as AJ_DEPTH blocks per multiprocessor remain.
template <typename T, bool GRAD>
cudaError_t run_words(WordsArgs a, bool streamed, int sms, cudaStream_t stream)
{
    const int named = GRAD ? 0 : a.r.n_bias;
    a.chunk = AJ_WORDS_CHUNK;
    while (a.chunk > 1024 && a.n_rows * ((a.vocab + a.chunk - 1) / a.chunk) < 4LL * sms) a.chunk /= 2;
    a.chunks = (a.vocab + a.chunk - 1) / a.chunk;
    a.entries = list_entries(a.r, named, a.chunk);
    int64_t rows = 1;
    if (a.r.history && a.r.share > 1 && named == 0 && a.mode != AJ_ALL_TOO) {
        rows = a.n_rows * a.chunks / ((int64_t)AJ_DEPTH * sms);
        rows = rows < 1 ? 1 : rows > AJ_ROWS ? AJ_ROWS : rows;
    }
    a.rows = (int)rows;
    const int64_t blocks = (a.n_rows + rows - 1) / rows * a.chunks;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    const bool half = a.r.history_len <= AJ_SHORT && named == 0 && a.mode != AJ_ALL_TOO;
    const int smem = half ? Table<true>::words(a.chunk, a.entries) * 4 : (four(Table<false>::words(a.chunk, a.entries)) + four(named) + named) * 4;
    void (*kernel)(WordsArgs) = half ? adjust_words_kernel<T, GRAD, true, false> : adjust_words_kernel<T, GRAD, false, false>;
    if constexpr (!GRAD) if (a.mode == AJ_ALL_TOO) kernel = adjust_words_kernel<T, false, false, true>;
    static std::atomic<unsigned long long> allowed[3];
    const cudaError_t e = allow_shared(kernel, AJ_MOST_SMEM, allowed[a.mode == AJ_ALL_TOO ? 2 : half]);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(half ? Table<true>::THREADS : Table<false>::THREADS);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = streamed ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T>
cudaError_t run_adjust(WordsArgs a, int sms, cudaStream_t stream)
{
    const bool place = a.logits == a.out, table = a.r.history || a.r.n_bias;
    a.other = Sixteen<T>::MINUS_INF;
    a.mode = !place || !table ? AJ_WORDS_ONLY : a.r.bias ? AJ_ALL_TOO : AJ_MASKED_TOO;
    const bool streamed = a.mode == AJ_WORDS_ONLY && (!place || a.r.bias || a.r.mask);
    if (streamed) {
        StreamArgs s = {};
        s.in = a.logits; s.out = a.out; s.bias = a.r.bias; s.mask = a.r.mask;
        s.in_stride = a.stride; s.out_stride = a.out_stride; s.bias_stride = a.r.bias_stride; s.mask_stride = a.r.mask_stride;
        s.n_rows = a.n_rows; s.vocab = a.vocab; s.other = a.other;
        int groups = 0;
        const cudaError_t e = run_stream<T>(s, sms, &groups, stream);
        if (e != cudaSuccess) return e;
    }
    return table ? run_words<T, false>(a, streamed, sms, stream) : cudaSuccess;
}

template <typename T>
cudaError_t run_adjust_grad(WordsArgs a, StreamArgs s, int sms, int* groups, cudaStream_t stream)
{
    const bool place = a.dout == a.out, table = a.r.history || a.dvalue;
    a.mode = !place || s.copy || s.partial || !a.r.history ? AJ_WORDS_ONLY : AJ_MASKED_TOO;
    const bool streamed = a.mode == AJ_WORDS_ONLY && (!place || s.copy || s.partial || s.mask);
    if (streamed) {
        const cudaError_t e = run_stream<T>(s, sms, groups, stream);
        if (e != cudaSuccess) return e;
    }
    return table ? run_words<T, true>(a, streamed, sms, stream) : cudaSuccess;
}

// The status of a call's launches.  A launch that failed leaves its error with the runtime, where the next call would take it for its own.
int launched(cudaError_t e)
{
    if (e == cudaSuccess) return APOLLO_OK;
    cudaGetLastError();
    return APOLLO_ERR_CUDA;
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
    WordsArgs a = {};
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
    return launched(err);
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
    WordsArgs a = {};
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
    if (a.r.history && d_grad_logits == d_logits && d_logits != d_grad_out) return APOLLO_ERR_INVALID_ARG;     // their signs are read beside the stream
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
    a.logits = d_logits; a.dout = d_grad_out; a.out = d_grad_logits; a.dvalue = a.r.n_bias ? d_grad_value : nullptr;
    a.stride = row_stride; a.dout_stride = grad_out_stride; a.out_stride = grad_logits_stride; a.n_rows = n_rows; a.vocab = (int)vocab;
    StreamArgs s = {};
    s.in = d_grad_out; s.out = d_grad_logits; s.copy = shared ? nullptr : d_grad_bias; s.partial = shared ? static_cast<float*>(d_workspace) : nullptr;
    s.mask = a.r.mask; s.in_stride = grad_out_stride; s.out_stride = grad_logits_stride; s.copy_stride = grad_bias_stride;
    s.mask_stride = a.r.mask_stride; s.n_rows = n_rows; s.vocab = (int)vocab;
    int groups = 0;
    cudaError_t err = dtype == APOLLO_DT_BF16 ? run_adjust_grad<__nv_bfloat16>(a, s, sms, &groups, stream) : run_adjust_grad<float>(a, s, sms, &groups, stream);
    if (err == cudaSuccess && shared) {
        const unsigned grid = (unsigned)((vocab + 31) / 32);
        if (dtype == APOLLO_DT_BF16) adjust_bias_join_kernel<<<grid, AJ_THREADS, 0, stream>>>(s.partial, groups, (int)vocab, static_cast<__nv_bfloat16*>(d_grad_bias));
        else adjust_bias_join_kernel<<<grid, AJ_THREADS, 0, stream>>>(s.partial, groups, (int)vocab, static_cast<float*>(d_grad_bias));
        err = cudaGetLastError();
    }
    return launched(err);
}
