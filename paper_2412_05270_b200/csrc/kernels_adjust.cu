// Logits adjusted by penalties for repeated tokens, biases and grammar masks, and the gradient of that.
//
//   c_j, d_j = occurrences of word j in the row's history, and from position `start` on
//   x = logit_j;  c_j > 0: x <- x > 0 ? x / rho : x rho;  d_j > 0: x <- x - (phi d_j + pi);  x <- x + bias_j + named values;
//   mask bit 0: x <- -inf
//   a_j = allowed ? dout_j : 0;  dlogit_j = a_j {1, 1 / rho, rho};  dbias_j = a_j (summed over rows if shared);  dvalue_i = a_j
//
// A CTA takes a chunk of the vocabulary of one row.  It reads the row's history and counts the tokens of its chunk in a table in
// shared memory (integer atomics: their order does not matter), then streams the chunk once.  A table word holds
// [31] seen at all  [30..20] 1 + slot of the word's named value  [19..0] how often from `start` on.
#include "../../include/apollo.h"

#include <cmath>

#include "device_utils.cuh"
#include "host_utils.h"

namespace apollo {

namespace {

constexpr int AJ_THREADS = 256;
constexpr int AJ_MAX_CHUNK = 8192;
constexpr int AJ_MIN_CHUNK = 2048;
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

// Counts the tokens of [j0, j0 + width) in the table (zeroed; a barrier before and after is the caller's).
__device__ __forceinline__ void count_history(const Rules& r, long long row, int vocab, int j0, int width, uint32_t* table)
{
    const long long first = row / r.share * r.history_stride;
    const int length = r.length ? min(max(r.length[row], 0), r.history_len) : r.history_len;
    const int start = r.start ? r.start[row] : 0;
    for (int i = threadIdx.x; i < length; i += AJ_THREADS) {
        const int j = token_at(r.history, first + i, r.history64, vocab) - j0;
        if (j >= 0 && j < width) {
            if (i >= start) atomicAdd(table + j, 1u);
            else atomicOr(table + j, AJ_SEEN);
        }
    }
}

template <typename T, int N> struct Vec;
template <typename T> struct Vec<T, 1> {
    T v;
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = (float)v; }
    __device__ __forceinline__ void set(const float (&x)[1]) { v = (T)x[0]; }
};
template <> struct Vec<float, 4> {
    float4 v;
    __device__ __forceinline__ void get(float (&x)[4]) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    __device__ __forceinline__ void set(const float (&x)[4]) { v = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Vec<__nv_bfloat16, 8> {
    uint4 v;
    __device__ __forceinline__ void get(float (&x)[8]) const { unpack_bf16x8(v, x); }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        v = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
};

template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, int count, float (&x)[N])
{
    if (count == N) reinterpret_cast<const Vec<T, N>*>(p)->get(x);
    else
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = e < count ? (float)p[e] : 0.0f;
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, int count, const float (&x)[N])
{
    if (count == N) {
        Vec<T, N> v;
        v.set(x);
        *reinterpret_cast<Vec<T, N>*>(p) = v;
    } else
#pragma unroll
        for (int e = 0; e < N; ++e) if (e < count) p[e] = (T)x[e];
}

// Mask bits of words j .. j + N - 1 (j a multiple of N, N a divisor of 32).
template <int N>
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* mask, int j)
{
    return mask ? mask[j >> 5] >> (j & 31) & ((1u << N) - 1u) : (1u << N) - 1u;
}

struct AdjustArgs {
    const void* logits;
    void* out;
    long long stride, out_stride, n_rows;
    int vocab, chunk;
    Rules r;
};

// N: elements of a vector; 1 where rows are not whole vectors.  TABLE: there is a history or there are named values.
template <typename T, int N, bool TABLE>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_kernel(const __grid_constant__ AdjustArgs a)
{
    extern __shared__ uint32_t table[];
    const int j0 = blockIdx.y * a.chunk, width = min(a.chunk, a.vocab - j0);
    float* sums = reinterpret_cast<float*>(table + a.chunk);
    int* words = reinterpret_cast<int*>(sums + a.r.n_bias);
    const bool place = a.logits == a.out;
    for (long long row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        float rho = 1.0f, phi = 0.0f, pi = 0.0f;
        if constexpr (TABLE) {
            __syncthreads();
            for (int i = threadIdx.x; i < width; i += AJ_THREADS) table[i] = 0;
            for (int i = threadIdx.x; i < a.r.n_bias; i += AJ_THREADS) words[i] = token_at(a.r.word, row * a.r.n_bias + i, a.r.words64, a.vocab);
            __syncthreads();
            if (a.r.history) {
                rho = a.r.rho_at ? a.r.rho_at[row] : a.r.rho;
                phi = a.r.phi_at ? a.r.phi_at[row] : a.r.phi;
                pi = a.r.pi_at ? a.r.pi_at[row] : a.r.pi;
                count_history(a.r, row, a.vocab, j0, width, table);
            }
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
                atomicOr(table + (w - j0), (uint32_t)(i + 1) << AJ_SLOT_SHIFT);
            }
            __syncthreads();
        }
        const T* x0 = static_cast<const T*>(a.logits) + row * a.stride;
        T* y0 = static_cast<T*>(a.out) + row * a.out_stride;
        const T* b0 = a.r.bias ? static_cast<const T*>(a.r.bias) + row * a.r.bias_stride : nullptr;
        const uint32_t* m0 = a.r.mask ? a.r.mask + row * a.r.mask_stride : nullptr;
        constexpr uint32_t ALL = (1u << N) - 1u;
        for (int u = threadIdx.x * N; u < width; u += AJ_THREADS * N) {
            const int j = j0 + u, count = min(N, width - u);
            const uint32_t live = mask_bits<N>(m0, j);
            uint32_t t[N], any = 0;
            if constexpr (TABLE) {
#pragma unroll
                for (int e = 0; e < N; ++e) { t[e] = e < count ? table[u + e] : 0; any |= t[e]; }
            }
            if (place && !b0 && any == 0 && live == ALL) continue;
            float x[N];
            if (live != 0) load_n<T, N>(x0 + j, count, x);
            if constexpr (TABLE) {
                if (any) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        if (t[e] & (AJ_SEEN | AJ_COUNT)) x[e] = x[e] > 0.0f ? __fdiv_rn(x[e], rho) : x[e] * rho;
                        if (t[e] & AJ_COUNT) x[e] -= fmaf(phi, (float)(t[e] & AJ_COUNT), pi);
                    }
                }
            }
            if (b0) {
                float b[N];
                load_n<T, N>(b0 + j, count, b);
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] += b[e];
            }
            if constexpr (TABLE) {
                if (any) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const uint32_t slot = t[e] >> AJ_SLOT_SHIFT & AJ_SLOT;
                        if (slot) x[e] += sums[slot - 1];
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) if (!(live >> e & 1)) x[e] = -INFINITY;
            store_n<T, N>(y0 + j, count, x);
        }
    }
}

struct AdjustGradArgs {
    const void* logits;
    const void* dout;
    void* dlogits;
    void* dbias;                         // rows of its own (dbias_stride > 0), or null
    float* partial;                      // shared bias: sums of a group of rows, vocab floats each
    float* dvalue;
    long long stride, dout_stride, dlogits_stride, dbias_stride, n_rows;
    int vocab, chunk, rows_per_group;
    Rules r;
};

// A CTA takes a chunk of the vocabulary for a group of rows; SUM: the sums over the group's rows stay in registers, UNITS vectors
// a thread.
template <typename T, int N, bool TABLE, bool SUM>
__global__ void __launch_bounds__(AJ_THREADS)
adjust_grad_kernel(const __grid_constant__ AdjustGradArgs a)
{
    constexpr int UNITS = SUM ? AJ_MIN_CHUNK / (AJ_THREADS * N) : 1;
    extern __shared__ uint32_t table[];
    const int j0 = blockIdx.y * a.chunk, width = min(a.chunk, a.vocab - j0);
    const bool place = a.dlogits == a.dout;
    const long long begin = (long long)blockIdx.x * a.rows_per_group, end = min(begin + a.rows_per_group, a.n_rows);
    float sum[UNITS][N];
#pragma unroll
    for (int k = 0; k < UNITS; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[k][e] = 0.0f;
    for (long long row = begin; row < end; ++row) {
        const T* x0 = static_cast<const T*>(a.logits) + row * a.stride;
        const T* g0 = static_cast<const T*>(a.dout) + row * a.dout_stride;
        T* y0 = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
        T* b0 = a.dbias ? static_cast<T*>(a.dbias) + row * a.dbias_stride : nullptr;
        const uint32_t* m0 = a.r.mask ? a.r.mask + row * a.r.mask_stride : nullptr;
        float rho = 1.0f;
        if constexpr (TABLE) {
            __syncthreads();
            for (int i = threadIdx.x; i < width; i += AJ_THREADS) table[i] = 0;
            __syncthreads();
            rho = a.r.rho_at ? a.r.rho_at[row] : a.r.rho;
            count_history(a.r, row, a.vocab, j0, width, table);
            __syncthreads();
        }
        if (a.dvalue) {
            // (in place: before anything of the row is overwritten)
            for (int i = threadIdx.x; i < a.r.n_bias; i += AJ_THREADS) {
                const int w = token_at(a.r.word, row * a.r.n_bias + i, a.r.words64, a.vocab);
                const bool none = w < 0;
                if (none ? j0 == 0 : w >= j0 && w < j0 + width)
                    a.dvalue[row * a.r.n_bias + i] = !none && (mask_bits<1>(m0, w) & 1u) ? (float)g0[w] : 0.0f;
            }
            if (place) __syncthreads();
        }
        constexpr uint32_t ALL = (1u << N) - 1u;
        int k = 0;
        for (int u = threadIdx.x * N; u < width; u += AJ_THREADS * N, ++k) {
            const int j = j0 + u, count = min(N, width - u);
            const uint32_t live = mask_bits<N>(m0, j);
            uint32_t t[N], any = 0;
            if constexpr (TABLE) {
#pragma unroll
                for (int e = 0; e < N; ++e) { t[e] = e < count ? table[u + e] : 0; any |= t[e]; }
            }
            if (!SUM && place && !b0 && any == 0 && live == ALL) continue;
            float g[N];
            if (live != 0) load_n<T, N>(g0 + j, count, g);
#pragma unroll
            for (int e = 0; e < N; ++e) if (!(live >> e & 1)) g[e] = 0.0f;
            if constexpr (SUM) {
#pragma unroll
                for (int q = 0; q < UNITS; ++q)
                    if (q == k)
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[q][e] += g[e];
            }
            if (b0) store_n<T, N>(b0 + j, count, g);
            if constexpr (TABLE) {
                if (any) {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (t[e] && (live >> e & 1)) g[e] = (float)x0[j + e] > 0.0f ? __fdiv_rn(g[e], rho) : g[e] * rho;
                }
            }
            if (!place || any || live != ALL) store_n<T, N>(y0 + j, count, g);
        }
    }
    if constexpr (SUM) {
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
            const int u = (k * AJ_THREADS + threadIdx.x) * N;
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (u + e < width) a.partial[(long long)blockIdx.x * a.vocab + j0 + u + e] = sum[k][e];
        }
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

constexpr int AJ_MAX_GROUPS = 256;

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

int pick_chunk(int64_t n_rows, int64_t vocab, int sms)
{
    int chunk = AJ_MAX_CHUNK;
    while (chunk > AJ_MIN_CHUNK && n_rows * ((vocab + chunk - 1) / chunk) < 4LL * sms) chunk /= 2;
    return chunk;
}

template <typename T, int N>
cudaError_t run_adjust(const AdjustArgs& a, cudaStream_t stream)
{
    const dim3 grid((unsigned)a.n_rows, (unsigned)((a.vocab + a.chunk - 1) / a.chunk));
    if (a.r.history || a.r.n_bias) adjust_kernel<T, N, true><<<grid, AJ_THREADS, (size_t)(a.chunk + 2 * a.r.n_bias) * 4, stream>>>(a);
    else adjust_kernel<T, N, false><<<grid, AJ_THREADS, 0, stream>>>(a);
    return cudaGetLastError();
}

template <typename T, int N>
cudaError_t run_adjust_grad(AdjustGradArgs a, int groups, cudaStream_t stream)
{
    const dim3 grid((unsigned)groups, (unsigned)((a.vocab + a.chunk - 1) / a.chunk));
    const size_t smem = a.r.history ? (size_t)a.chunk * 4 : 0;
    if (a.partial) {
        if (a.r.history) adjust_grad_kernel<T, N, true, true><<<grid, AJ_THREADS, smem, stream>>>(a);
        else adjust_grad_kernel<T, N, false, true><<<grid, AJ_THREADS, smem, stream>>>(a);
    } else {
        if (a.r.history) adjust_grad_kernel<T, N, true, false><<<grid, AJ_THREADS, smem, stream>>>(a);
        else adjust_grad_kernel<T, N, false, false><<<grid, AJ_THREADS, smem, stream>>>(a);
    }
    return cudaGetLastError();
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
    a.chunk = pick_chunk(n_rows, vocab, sms);
    const bool vec = whole_vectors(d_logits, row_stride, e) && whole_vectors(d_out, out_stride, e) && whole_vectors(a.r.bias, a.r.bias_stride, e);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (dtype == APOLLO_DT_BF16) err = vec ? run_adjust<__nv_bfloat16, 8>(a, stream) : run_adjust<__nv_bfloat16, 1>(a, stream);
    else err = vec ? run_adjust<float, 4>(a, stream) : run_adjust<float, 1>(a, stream);
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
    a.chunk = shared ? AJ_MIN_CHUNK : pick_chunk(n_rows, vocab, sms);
    a.rows_per_group = shared ? (int)((n_rows + AJ_MAX_GROUPS - 1) / AJ_MAX_GROUPS) : 1;
    const int groups = (int)((n_rows + a.rows_per_group - 1) / a.rows_per_group);
    const bool vec = whole_vectors(d_grad_out, grad_out_stride, e) && whole_vectors(d_grad_logits, grad_logits_stride, e) &&
                     whole_vectors(a.dbias, a.dbias ? grad_bias_stride : 0, e);
    cudaError_t err;
    if (dtype == APOLLO_DT_BF16) err = vec ? run_adjust_grad<__nv_bfloat16, 8>(a, groups, stream) : run_adjust_grad<__nv_bfloat16, 1>(a, groups, stream);
    else err = vec ? run_adjust_grad<float, 4>(a, groups, stream) : run_adjust_grad<float, 1>(a, groups, stream);
    if (err == cudaSuccess && shared) {
        const unsigned grid = (unsigned)((vocab + AJ_THREADS - 1) / AJ_THREADS);
        if (dtype == APOLLO_DT_BF16) adjust_bias_join_kernel<<<grid, AJ_THREADS, 0, stream>>>(a.partial, groups, (int)vocab, static_cast<__nv_bfloat16*>(d_grad_bias));
        else adjust_bias_join_kernel<<<grid, AJ_THREADS, 0, stream>>>(a.partial, groups, (int)vocab, static_cast<float*>(d_grad_bias));
        err = cudaGetLastError();
    }
    return err == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}
