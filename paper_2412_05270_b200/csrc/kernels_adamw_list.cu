// The global norm of a list of gradients with the factor that clips it, and AdamW over a list of tensors of mixed types with
// moments of 8 or 32 bits: the step for everything that the method does not project, in one launch per pair of types.
//
//   norm = sqrt(sum G^2),  factor = min(1, max_norm / norm)
//   g = factor G,  m <- b1 m + (1-b1) g,  v <- b2 v + (1-b2) g^2,  P <- P - lr ((m / c1) / (sqrt(v / c2) + eps) + wd P)
//
// 8-bit moments.  Blocks of 256 elements (one per warp, eight elements a lane) share an exponent byte k per moment.  A code c is
// the float whose bits are (c << 20) + (k << 23): exponent and three mantissa bits, counted from the block's own exponent.  So
// decoding is a shift and an add, and rounding x stochastically is (bits(x) + r) >> 20 with r uniform in [0, 2^20): the sum
// carries with the probability that the 20 cut bits stand for.  No value leaves the range on either side: k is taken from the
// largest element, rounded up before its exponent is read, and covers every exponent of fp32.
//   m: sign and 7 bits, 16 binades below the largest, code 0 is zero.
//   v: 8 bits, 32 binades (as wide as m's 16, as sqrt(v) goes); code 0 is the lowest value, not zero, so an element whose v falls
//      below it is not divided by eps.
// Why stochastic: v moves by (1-b2) = 1/1000 of itself a step and the codes are 6 to 12 % apart; rounded to nearest it would
// never move (m likewise once g is within 60 % of it).  16 random bits per element: a probability of 1/100 then is right to
// 0.2 %.  One Philox4x32-10 call a lane gives the 128 bits that its eight elements need; m and v share them (each is unbiased,
// and errors of the same sign cancel in m / sqrt(v)).
#include "../../include/apollo.h"

#include <cmath>

#include "device_utils.cuh"
#include "host_utils.h"
#include "philox.cuh"
#include "tc_ptx.cuh"

namespace apollo {

namespace {

constexpr int AL_BLOCK = APOLLO_ADAMW_BLOCK;
constexpr int AL_THREADS = 256;
constexpr int AL_WARPS = AL_THREADS / 32;
constexpr int AL_TILE = 32;              // blocks of one tile: four for each warp
constexpr int AL_FEW = 48, AL_MANY = 960;   // tensors whose pointers travel as parameters of one launch (CUDA: 32,764 bytes)

__device__ __forceinline__ void store8(float* p, const float (&v)[8])
{
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8])
{
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// ---------------------------------------------------------------- norm
constexpr int GN_TILE = 8192;            // elements of one tile
constexpr int GN_THREADS = 256;
constexpr int GN_MAX_GRID = 2048;        // partial sums of one launch at most

template <int CAP>
struct NormArgs {
    const void* g[CAP];
    long long numel[CAP];
    int tile_begin[CAP + 1];
    unsigned char bf16[CAP];
    int n;
    double* partial;
};

// Sum of the squares of eight raw 16-byte vectors (a thread's share of a tile is 32 elements of either type).
template <typename T> struct NormShare;
template <> struct NormShare<__nv_bfloat16> { static constexpr int VECS = 4, N = 8; };
template <> struct NormShare<float> { static constexpr int VECS = 8, N = 4; };

__device__ __forceinline__ void norm_unpack(const uint4& r, float (&v)[8], __nv_bfloat16) { unpack_bf16x8(r, v); }
__device__ __forceinline__ void norm_unpack(const uint4& r, float (&v)[4], float)
{
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
}

template <typename T>
__device__ __forceinline__ double tile_squares(const T* __restrict__ g, long long numel, long long e0)
{
    constexpr int VECS = NormShare<T>::VECS, N = NormShare<T>::N;
    uint4 raw[VECS];
    if (e0 + GN_TILE <= numel) {
#pragma unroll
        for (int i = 0; i < VECS; ++i) raw[i] = __ldcs(reinterpret_cast<const uint4*>(g + e0) + i * GN_THREADS + threadIdx.x);
    } else {
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const long long e = e0 + (long long)(i * GN_THREADS + threadIdx.x) * N;
            if (e + N <= numel) {
                raw[i] = __ldcs(reinterpret_cast<const uint4*>(g + e));
            } else {
                uint32_t w[4] = { 0, 0, 0, 0 };
                for (int x = 0; x < N; ++x)
                    if (e + x < numel) {
                        if (sizeof(T) == 4) w[x & 3] = __float_as_uint(load1(g + e + x));
                        else w[(x >> 1) & 3] |= (uint32_t)reinterpret_cast<const unsigned short*>(g)[e + x] << (16 * (x & 1));
                    }
                raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        float v[N];
        norm_unpack(raw[i], v, T());
#pragma unroll
        for (int x = 0; x < N; ++x) s = fmaf(v[x], v[x], s);
    }
    // In the middle of fp32's range nothing has overflowed, and what may have underflowed is below 2^-36 of the sum.
    if (s >= 0x1p-90f && s <= 0x1p120f) return (double)s;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) any |= raw[i].x | raw[i].y | raw[i].z | raw[i].w;
    if (any == 0) return 0.0;
    double d = 0.0;
#pragma unroll 1
    for (int i = 0; i < VECS; ++i) {
        float v[N];
        uint4 r = raw[0];
#pragma unroll
        for (int k = 1; k < VECS; ++k) if (k == i) r = raw[k];
        norm_unpack(r, v, T());
#pragma unroll
        for (int x = 0; x < N; ++x) d += (double)v[x] * (double)v[x];
    }
    return d;
}

template <int CAP>
__global__ void __launch_bounds__(GN_THREADS)
grad_norm_kernel(const __grid_constant__ NormArgs<CAP> a)
{
    __shared__ double scratch[32];
    ptx::grid_launch_dependents();
    double sum = 0.0;
    const int tiles = a.tile_begin[a.n];
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int lo = 0, hi = a.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.tile_begin[mid] <= tile) lo = mid; else hi = mid;
        }
        const long long e0 = (long long)(tile - a.tile_begin[lo]) * GN_TILE;
        sum += a.bf16[lo] ? tile_squares(static_cast<const __nv_bfloat16*>(a.g[lo]), a.numel[lo], e0)
                          : tile_squares(static_cast<const float*>(a.g[lo]), a.numel[lo], e0);
    }
    const double total = block_sum(sum, scratch);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = total;
}

__global__ void __launch_bounds__(GN_THREADS)
grad_norm_join_kernel(const double* __restrict__ partial, int n, double max_norm, float* __restrict__ out)
{
    __shared__ double scratch[32];
    ptx::grid_wait_previous();
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += GN_THREADS) sum += partial[i];
    const double total = block_sum(sum, scratch);
    if (threadIdx.x == 0) {
        const double norm = sqrt(total);
        out[0] = (float)norm;
        out[1] = !isfinite(norm) ? __int_as_float(0x7FFFFFFF) : norm > max_norm ? (float)(max_norm / norm) : 1.0f;
    }
}

// ---------------------------------------------------------------- step
template <int CAP>
struct ListArgs {
    void* p[CAP];
    const void* g[CAP];
    long long numel[CAP];
    int tile_begin[CAP + 1];
    int block_begin[CAP];                // the tensor's first block in the state
    int n;
    char* m;                             // 8 bits: codes; 32 bits: floats
    char* v;
    uint16_t* k;                         // 8 bits: m's exponent, v's exponent << 8
    const float* factor;
    const float* lr_at;
    const long long* t_at;
    float lr, wd, eps, b1, a1, b2, a2;   // a = 1 - b
    float inv_c1, inv_c2;
    double log_b1, log_b2;               // for the step count on the device
    int bias_correction;
    unsigned long long t;
    uint32_t keys[20];
};

struct Scalars { float lr, factor, inv_c1, inv_c2; uint32_t t_lo, t_hi; };

// Exponent byte of a block whose largest magnitude has these bits, for codes of TOP + 1 binades.
template <int TOP>
__device__ __forceinline__ int exponent_of(uint32_t largest)
{
    const int e = (int)((largest + 0xFFFFFu) >> 23) - TOP;
    return min(max(e, 0), 255 - TOP);
}

template <typename PT, typename GT, bool Q8, int CAP>
__global__ void __launch_bounds__(AL_THREADS)
adamw_list_kernel(const __grid_constant__ ListArgs<CAP> a)
{
    __shared__ Scalars shared;
    if (threadIdx.x == 0) {
        Scalars s;
        s.lr = a.lr_at ? *a.lr_at : a.lr;
        s.factor = a.factor ? *a.factor : 1.0f;
        unsigned long long t = a.t;
        s.inv_c1 = a.inv_c1; s.inv_c2 = a.inv_c2;
        if (a.t_at) {
            t = (unsigned long long)*a.t_at;
            if (a.bias_correction) {
                s.inv_c1 = (float)(-1.0 / expm1((double)(t + 1) * a.log_b1));
                s.inv_c2 = (float)(-1.0 / expm1((double)(t + 1) * a.log_b2));
            }
        }
        s.t_lo = (uint32_t)t; s.t_hi = (uint32_t)(t >> 32);
        shared = s;
    }
    __syncthreads();
    const Scalars s = shared;
    if (!isfinite(s.factor)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tiles = a.tile_begin[a.n];
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int at = 0, hi = a.n;
        while (hi - at > 1) {
            const int mid = (at + hi) >> 1;
            if (a.tile_begin[mid] <= tile) at = mid; else hi = mid;
        }
        PT* __restrict__ P = static_cast<PT*>(a.p[at]);
        const GT* __restrict__ G = static_cast<const GT*>(a.g[at]);
        const long long numel = a.numel[at];
        const int first = (tile - a.tile_begin[at]) * AL_TILE + warp;
        for (int i = 0; i < AL_TILE / AL_WARPS; ++i) {
            const int local = first + i * AL_WARPS;
            const long long e = (long long)local * AL_BLOCK + lane * 8;
            if (e - lane * 8 >= numel) break;
            const int block = a.block_begin[at] + local;
            const long long se = (long long)block * AL_BLOCK + lane * 8;
            const int count = (int)max(0ll, min(8ll, numel - e));
            float g[8], p[8], m[8], v[8];
            if (count == 8) { load8_stream(G + e, g); load8_stream(P + e, p); }
            else { load8_guarded(G + e, count, g); load8_guarded(P + e, count, p); }
            if constexpr (Q8) {
                const uint2 cm = __ldcs(reinterpret_cast<const uint2*>(a.m + se)), cv = __ldcs(reinterpret_cast<const uint2*>(a.v + se));
                const uint32_t k = a.k[block];
                const uint32_t km = (k & 255u) << 23, kv = (k >> 8) << 23;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint32_t bm = ((x < 4 ? cm.x : cm.y) >> (8 * (x & 3))) & 255u, bv = ((x < 4 ? cv.x : cv.y) >> (8 * (x & 3))) & 255u;
                    const uint32_t mag = bm & 127u;
                    m[x] = __uint_as_float((mag ? (mag << 20) + km : 0u) | (bm & 128u) << 24);
                    v[x] = __uint_as_float((bv << 20) + kv);
                }
            } else {
                const float* M = reinterpret_cast<const float*>(a.m) + se;
                const float* V = reinterpret_cast<const float*>(a.v) + se;
                if (count == 8) { load8_stream(M, m); load8_stream(V, v); }
                else { load8_guarded(M, count, m); load8_guarded(V, count, v); }
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const float gx = g[x] * s.factor;
                m[x] = fmaf(a.b1, m[x], a.a1 * gx);
                v[x] = fmaf(a.b2, v[x], a.a2 * gx * gx);
                const float update = __fdividef(m[x] * s.inv_c1, sqrtf(v[x] * s.inv_c2) + a.eps);
                p[x] = fmaf(-s.lr, fmaf(a.wd, p[x], update), p[x]);
            }
            if (count == 8) store8(P + e, p);
            else for (int x = 0; x < count; ++x) store1(P + e + x, p[x]);
            if constexpr (Q8) {
                uint32_t top_m = 0, top_v = 0;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    top_m = max(top_m, __float_as_uint(m[x]) & 0x7FFFFFFFu);
                    top_v = max(top_v, __float_as_uint(v[x]));
                }
                const int km = exponent_of<15>(__reduce_max_sync(0xFFFFFFFFu, top_m)), kv = exponent_of<31>(__reduce_max_sync(0xFFFFFFFFu, top_v));
                const uint4 r4 = philox4x32_10_keys((uint32_t)block, (uint32_t)lane, s.t_lo, s.t_hi, a.keys);
                const uint32_t r[4] = { r4.x, r4.y, r4.z, r4.w };
                uint32_t cm[2] = { 0, 0 }, cv[2] = { 0, 0 };
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint32_t dither = (x & 1 ? r[x >> 1] >> 16 : r[x >> 1] & 0xFFFFu) << 4;
                    const uint32_t bits = __float_as_uint(m[x]);
                    const int em = min(max((int)(((bits & 0x7FFFFFFFu) + dither) >> 20) - km * 8, 0), 127);
                    const int ev = min(max((int)((__float_as_uint(v[x]) + dither) >> 20) - kv * 8, 0), 255);
                    cm[x >> 2] |= ((uint32_t)em | (bits >> 24 & 128u)) << (8 * (x & 3));
                    cv[x >> 2] |= (uint32_t)ev << (8 * (x & 3));
                }
                __stcs(reinterpret_cast<uint2*>(a.m + se), make_uint2(cm[0], cm[1]));
                __stcs(reinterpret_cast<uint2*>(a.v + se), make_uint2(cv[0], cv[1]));
                if (lane == 0) a.k[block] = (uint16_t)(km | kv << 8);
            } else {
                float* M = reinterpret_cast<float*>(a.m) + se;
                float* V = reinterpret_cast<float*>(a.v) + se;
                if (count == 8) { store8(M, m); store8(V, v); }
                else for (int x = 0; x < count; ++x) { M[x] = m[x]; V[x] = v[x]; }
            }
        }
    }
}

// Values of 8-bit moments, sixteen elements a thread.
__global__ void __launch_bounds__(AL_THREADS)
adamw_moments_kernel(const uint4* __restrict__ cm, const uint4* __restrict__ cv, const uint16_t* __restrict__ ks, long long n,
                     uint4* __restrict__ m, uint4* __restrict__ v)
{
    for (long long i = (long long)blockIdx.x * AL_THREADS + threadIdx.x; i < n; i += (long long)gridDim.x * AL_THREADS) {
        const uint4 m4 = __ldcs(cm + i), v4 = __ldcs(cv + i);
        const uint32_t k = __ldg(ks + (i >> 4)), km = (k & 255u) << 7, kv = (k >> 8) << 7;
        const uint32_t mw[4] = { m4.x, m4.y, m4.z, m4.w }, vw[4] = { v4.x, v4.y, v4.z, v4.w };
        uint32_t mo[8], vo[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {        // bfloat16 is the upper half of the float: (c << 4) + (k << 7)
            uint32_t h[2], u[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int sh = 8 * ((2 * x + y) & 3);
                const uint32_t bm = (mw[x >> 1] >> sh) & 255u, mag = bm & 127u;
                h[y] = (mag ? (mag << 4) + km : 0u) | (bm & 128u) << 8;
                u[y] = (((vw[x >> 1] >> sh) & 255u) << 4) + kv;
            }
            mo[x] = h[0] | h[1] << 16;
            vo[x] = u[0] | u[1] << 16;
        }
        __stcs(m + 2 * i, make_uint4(mo[0], mo[1], mo[2], mo[3])); __stcs(m + 2 * i + 1, make_uint4(mo[4], mo[5], mo[6], mo[7]));
        __stcs(v + 2 * i, make_uint4(vo[0], vo[1], vo[2], vo[3])); __stcs(v + 2 * i + 1, make_uint4(vo[4], vo[5], vo[6], vo[7]));
    }
}

bool known_dtype(int32_t d) { return d == APOLLO_DT_F32 || d == APOLLO_DT_BF16; }

// Blocks of a list, or -1 where they pass 2^31 - 1.
int64_t count_blocks(const int64_t* numel, int32_t n)
{
    int64_t blocks = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] > (int64_t)INT32_MAX * AL_BLOCK) return -1;
        blocks += (numel[i] + AL_BLOCK - 1) / AL_BLOCK;
        if (blocks > INT32_MAX) return -1;
    }
    return blocks;
}

size_t state_size(int64_t blocks, int32_t bits) { return bits == 32 ? (size_t)blocks * AL_BLOCK * 8 : (size_t)blocks * (AL_BLOCK * 2 + 2); }

int norm_grid(int64_t tiles, int sms)
{
    const int64_t most = 8LL * sms < GN_MAX_GRID ? 8LL * sms : GN_MAX_GRID;
    return (int)(tiles < most ? tiles : most);
}

// One launch over the tensors order[0 .. count): the sums of its blocks to partial[0 .. *blocks).
template <int CAP>
int norm_launch(const void* const* d_G, const int64_t* numel, const int32_t* dtype, const int32_t* order, int32_t count, double* partial,
                int sms, cudaStream_t stream, int* blocks)
{
    NormArgs<CAP> a;
    int64_t tiles = 0;
    for (int k = 0; k < count; ++k) {
        const int i = order[k];
        a.g[k] = d_G[i]; a.numel[k] = numel[i]; a.bf16[k] = dtype[i] == APOLLO_DT_BF16;
        a.tile_begin[k] = (int)tiles;
        tiles += (numel[i] + GN_TILE - 1) / GN_TILE;
        if (tiles > INT32_MAX) return APOLLO_ERR_SHAPE;
    }
    a.tile_begin[count] = (int)tiles;
    a.n = count; a.partial = partial;
    *blocks = norm_grid(tiles, sms);
    grad_norm_kernel<CAP><<<*blocks, GN_THREADS, 0, stream>>>(a);
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}

template <typename PT, typename GT, bool Q8, int CAP>
cudaError_t list_launch(const ListArgs<CAP>& a, int64_t tiles, int sms, cudaStream_t stream)
{
    const int64_t most = 8LL * sms;
    adamw_list_kernel<PT, GT, Q8, CAP><<<(unsigned)(tiles < most ? tiles : most), AL_THREADS, 0, stream>>>(a);
    return cudaGetLastError();
}

struct ListCall {
    void* const* P;
    const void* const* G;
    const int64_t* numel;
    const int32_t *dtype_P, *dtype_G;
    int32_t n;
    bool q8;
    int sms;
    cudaStream_t stream;
};

// The tensors of one pair of types, CAP at a time.
template <int CAP>
int list_launches(const ListCall& c, ListArgs<CAP>& a, int32_t dp, int32_t dg)
{
    int64_t block = 0, tiles = 0;
    a.n = 0;
    for (int32_t i = 0; i <= c.n; ++i) {
        if ((i == c.n || a.n == CAP) && a.n > 0) {
            a.tile_begin[a.n] = (int)tiles;
            const bool pb = dp == APOLLO_DT_BF16, gb = dg == APOLLO_DT_BF16;
            cudaError_t e;
            if (c.q8)
                e = pb ? (gb ? list_launch<__nv_bfloat16, __nv_bfloat16, true>(a, tiles, c.sms, c.stream) : list_launch<__nv_bfloat16, float, true>(a, tiles, c.sms, c.stream))
                       : (gb ? list_launch<float, __nv_bfloat16, true>(a, tiles, c.sms, c.stream) : list_launch<float, float, true>(a, tiles, c.sms, c.stream));
            else
                e = pb ? (gb ? list_launch<__nv_bfloat16, __nv_bfloat16, false>(a, tiles, c.sms, c.stream) : list_launch<__nv_bfloat16, float, false>(a, tiles, c.sms, c.stream))
                       : (gb ? list_launch<float, __nv_bfloat16, false>(a, tiles, c.sms, c.stream) : list_launch<float, float, false>(a, tiles, c.sms, c.stream));
            if (e != cudaSuccess) return APOLLO_ERR_CUDA;
            a.n = 0;
            tiles = 0;
        }
        if (i == c.n) break;
        const int64_t blocks = (c.numel[i] + AL_BLOCK - 1) / AL_BLOCK;
        if (c.G[i] && blocks > 0 && c.dtype_P[i] == dp && c.dtype_G[i] == dg) {
            a.p[a.n] = c.P[i]; a.g[a.n] = c.G[i]; a.numel[a.n] = c.numel[i];
            a.tile_begin[a.n] = (int)tiles; a.block_begin[a.n] = (int)block;
            tiles += (blocks + AL_TILE - 1) / AL_TILE;
            ++a.n;
        }
        block += blocks;
    }
    return APOLLO_OK;
}

template <int CAP>
int list_step(const ListCall& c, const apollo_adamw_list_config* cfg, void* d_state, int64_t blocks, double lr, double wd, int64_t t,
              const float* d_factor, const float* d_lr, const int64_t* d_t)
{
    ListArgs<CAP> a;
    const size_t codes = (size_t)blocks * AL_BLOCK * (c.q8 ? 1 : 4);
    a.m = static_cast<char*>(d_state); a.v = a.m + codes; a.k = reinterpret_cast<uint16_t*>(a.v + codes);
    a.factor = d_factor; a.lr_at = d_lr; a.t_at = reinterpret_cast<const long long*>(d_t);
    a.lr = (float)lr; a.wd = (float)wd; a.eps = (float)cfg->eps;
    a.b1 = (float)cfg->beta1; a.a1 = (float)(1.0 - cfg->beta1); a.b2 = (float)cfg->beta2; a.a2 = (float)(1.0 - cfg->beta2);
    a.bias_correction = cfg->bias_correction;
    a.log_b1 = std::log(cfg->beta1); a.log_b2 = std::log(cfg->beta2);      // (-inf for 0: expm1 is -1, c = 1)
    a.inv_c1 = a.inv_c2 = 1.0f;
    if (cfg->bias_correction) {
        a.inv_c1 = (float)(-1.0 / std::expm1(((double)t + 1) * a.log_b1));
        a.inv_c2 = (float)(-1.0 / std::expm1(((double)t + 1) * a.log_b2));
    }
    a.t = (unsigned long long)t;
    uint32_t k0 = (uint32_t)cfg->seed, k1 = (uint32_t)(cfg->seed >> 32);
    for (int r = 0; r < 10; ++r) {
        a.keys[2 * r] = k0; a.keys[2 * r + 1] = k1;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    for (int32_t dp = 0; dp < 2; ++dp)
        for (int32_t dg = 0; dg < 2; ++dg) {
            const int rc = list_launches<CAP>(c, a, dp, dg);
            if (rc != APOLLO_OK) return rc;
        }
    return APOLLO_OK;
}

}  // namespace

}  // namespace apollo

using namespace apollo;

extern "C" int apollo_grad_norm_workspace_bytes(int32_t n_tensors, size_t* out_bytes)
{
    if (!out_bytes || n_tensors < 1) return APOLLO_ERR_INVALID_ARG;
    *out_bytes = ((size_t)n_tensors + AL_MANY - 1) / AL_MANY * GN_MAX_GRID * sizeof(double);
    return APOLLO_OK;
}

extern "C" int apollo_grad_norm(const void* const* d_G, const int64_t* numel, const int32_t* dtype, int32_t n_tensors,
                                double max_norm, float* d_out, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    size_t need = 0;
    const int rc = apollo_grad_norm_workspace_bytes(n_tensors, &need);
    if (rc != APOLLO_OK) return rc;
    if (!d_G || !numel || !dtype || !d_out || !d_workspace || !(max_norm > 0.0)) return APOLLO_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (!known_dtype(dtype[i]) || numel[i] < 0) return APOLLO_ERR_INVALID_ARG;
        if (numel[i] > (int64_t)INT32_MAX * GN_TILE) return APOLLO_ERR_SHAPE;
        if ((uintptr_t)d_G[i] % 16) return APOLLO_ERR_ALIGN;
    }
    if ((uintptr_t)d_out % 4 || (uintptr_t)d_workspace % 16) return APOLLO_ERR_ALIGN;
    if (workspace_bytes < need) return APOLLO_ERR_WORKSPACE;
    int sms = 0;
    const int drc = device_sms(&sms);
    if (drc != APOLLO_OK) return drc;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    double* partial = static_cast<double*>(d_workspace);
    int32_t order[AL_MANY];
    int32_t count = 0, total = 0;
    for (int32_t i = 0; i <= n_tensors; ++i) {
        if (count > 0 && (i == n_tensors || count == AL_MANY)) {
            int blocks = 0;
            const int lrc = count <= AL_FEW ? norm_launch<AL_FEW>(d_G, numel, dtype, order, count, partial + total, sms, stream, &blocks)
                                            : norm_launch<AL_MANY>(d_G, numel, dtype, order, count, partial + total, sms, stream, &blocks);
            if (lrc != APOLLO_OK) { cudaGetLastError(); return lrc; }
            total += blocks;
            count = 0;
        }
        if (i < n_tensors && d_G[i] && numel[i] > 0) order[count++] = i;
    }
    if (total == 0) grad_norm_join_kernel<<<1, GN_THREADS, 0, stream>>>(partial, 0, max_norm, d_out);
    else launch_after(grad_norm_join_kernel, dim3(1), dim3(GN_THREADS), stream, (const double*)partial, (int)total, max_norm, d_out);
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}

extern "C" int apollo_adamw_list_state_bytes(const int64_t* numel, int32_t n_tensors, int32_t state_bits, size_t* out_bytes)
{
    if (!numel || !out_bytes || n_tensors < 1 || (state_bits != 8 && state_bits != 32)) return APOLLO_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_tensors; ++i)
        if (numel[i] < 0) return APOLLO_ERR_INVALID_ARG;
    const int64_t blocks = count_blocks(numel, n_tensors);
    if (blocks < 0) return APOLLO_ERR_SHAPE;
    *out_bytes = state_size(blocks, state_bits);
    return APOLLO_OK;
}

extern "C" int apollo_adamw_list_step(const apollo_adamw_list_config* cfg, void* const* d_P, const void* const* d_G,
                                      const int64_t* numel, const int32_t* dtype_P, const int32_t* dtype_G, int32_t n_tensors,
                                      void* d_state, size_t state_bytes, double lr, double wd, int64_t t, const float* d_factor,
                                      const float* d_lr, const int64_t* d_t, void* cuda_stream)
{
    if (!cfg || !d_P || !d_G || !dtype_P || !dtype_G) return APOLLO_ERR_INVALID_ARG;
    size_t need = 0;
    const int rc = apollo_adamw_list_state_bytes(numel, n_tensors, cfg->state_bits, &need);
    if (rc != APOLLO_OK) return rc;
    if (!std::isfinite(lr) || !std::isfinite(wd) || !std::isfinite(cfg->eps) || cfg->eps < 0.0 || t < 0) return APOLLO_ERR_INVALID_ARG;
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return APOLLO_ERR_INVALID_ARG;
    if (cfg->bias_correction != 0 && cfg->bias_correction != 1) return APOLLO_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (!known_dtype(dtype_P[i]) || !known_dtype(dtype_G[i])) return APOLLO_ERR_INVALID_ARG;
        if (!d_P[i] && d_G[i] && numel[i] > 0) return APOLLO_ERR_INVALID_ARG;
        if ((uintptr_t)d_P[i] % 16 || (uintptr_t)d_G[i] % 16) return APOLLO_ERR_ALIGN;
    }
    if (need > 0 && !d_state) return APOLLO_ERR_INVALID_ARG;
    if ((uintptr_t)d_state % 16 || (uintptr_t)d_factor % 4 || (uintptr_t)d_lr % 4 || (uintptr_t)d_t % 8) return APOLLO_ERR_ALIGN;
    if (state_bytes < need) return APOLLO_ERR_WORKSPACE;
    ListCall c{ d_P, d_G, numel, dtype_P, dtype_G, n_tensors, cfg->state_bits == 8, 0, static_cast<cudaStream_t>(cuda_stream) };
    const int drc = device_sms(&c.sms);
    if (drc != APOLLO_OK) return drc;
    const int64_t blocks = count_blocks(numel, n_tensors);
    const int src = n_tensors <= AL_FEW ? list_step<AL_FEW>(c, cfg, d_state, blocks, lr, wd, t, d_factor, d_lr, d_t)
                                        : list_step<AL_MANY>(c, cfg, d_state, blocks, lr, wd, t, d_factor, d_lr, d_t);
    if (src != APOLLO_OK) cudaGetLastError();
    return src;
}

extern "C" int apollo_adamw_list_moments(const void* d_state, size_t state_bytes, int64_t n_blocks, void* d_M, void* d_V, void* cuda_stream)
{
    if (n_blocks < 0) return APOLLO_ERR_INVALID_ARG;
    if (n_blocks > INT32_MAX) return APOLLO_ERR_SHAPE;
    if (n_blocks == 0) return APOLLO_OK;
    if (!d_state || !d_M || !d_V) return APOLLO_ERR_INVALID_ARG;
    if ((uintptr_t)d_state % 16 || (uintptr_t)d_M % 16 || (uintptr_t)d_V % 16) return APOLLO_ERR_ALIGN;
    if (state_bytes < state_size(n_blocks, 8)) return APOLLO_ERR_WORKSPACE;
    int sms = 0;
    const int drc = device_sms(&sms);
    if (drc != APOLLO_OK) return drc;
    const char* m = static_cast<const char*>(d_state);
    const char* v = m + (size_t)n_blocks * AL_BLOCK;
    const int64_t vectors = n_blocks * (AL_BLOCK / 16), most = 8LL * sms;
    const int64_t grid = (vectors + AL_THREADS - 1) / AL_THREADS;
    adamw_moments_kernel<<<(unsigned)(grid < most ? grid : most), AL_THREADS, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        reinterpret_cast<const uint4*>(m), reinterpret_cast<const uint4*>(v), reinterpret_cast<const uint16_t*>(v + (size_t)n_blocks * AL_BLOCK),
        vectors, static_cast<uint4*>(d_M), static_cast<uint4*>(d_V));
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}
