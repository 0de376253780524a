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
// 0.2 %.  One Philox4x32-10 call a lane gives the 128 bits that its eight elements need; m and v share them (errors of the same sign
// cancel in m / sqrt(v)).  Rounding is unbiased from code 1 on.  Below it an m is rounded as if code 0 were the power of two under code 1, but held
// as zero, and an m below that power (about 2^-15 of its block's largest) is zero every time (it has its part in the update before);
// a v below code 0 is raised to it.
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
constexpr int AL_TILE32 = 4096;          // elements of one tile, 32 bits
constexpr int AL_WAVES = 16;             // 8 bits: how many times the blocks that are resident at once, at most
// Tensors whose pointers travel as parameters of one launch: as many as fit CUDA's 32,764 bytes, or few, which launch faster.
constexpr int AL_FEW = 96, AL_MANY = 960;

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
// One read of every gradient, squares and sums in fp64: the norm is rounded once.  262 M bfloat16 in 87 us, 6.0 TB/s; fp32 in 152 us, 6.9 TB/s.
// (32 squares at a time in fp32: 81 us, but squares of bfloat16 end in few bit patterns, so the rounding of their sums is biased: 1e-8 of the
// norm, one seed in eight had another last bit, and with the factor's last bit a clipped step has other codes.  Values converted by cvt instead of
// moved bits: 90.5 us.  The next tile's loads under way in registers: 81 us, but fp32 154 to 162, and a 60M model's gradients 27 us either way.)
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

// A thread's share of a tile is 32 elements of either type, in vectors of 16 bytes.  squares() adds up those of a word (one fp32, two bfloat16) times
// 2^-256: the bits of |v| moved to a double's place, with an exponent that makes it 2^-128 |v|.  Zero becomes 2^-255 instead, a subnormal number
// 2^-255 to 2^-254, infinity and NaN at least 1: sums outside [2^-436, 1) are formed once more from converted values.
template <typename T> struct NormShare;
template <> struct NormShare<__nv_bfloat16> {
    static constexpr int VECS = 4, N = 8;
    static constexpr uint32_t MAGNITUDE = 0x7FFF7FFFu;
    __device__ static __forceinline__ double moved(uint32_t h) { return __hiloint2double((int)((h & 0x0FFFE000u) | 0x30000000u), 0); }
    __device__ static __forceinline__ void squares(uint32_t w, double& s, double& t)
    {
        const double a = moved(w << 13), b = moved(w >> 3);
        s = fma(a, a, s);
        t = fma(b, b, t);
    }
};
template <> struct NormShare<float> {
    static constexpr int VECS = 8, N = 4;
    static constexpr uint32_t MAGNITUDE = 0x7FFFFFFFu;
    __device__ static __forceinline__ void squares(uint32_t w, double& s, double&)
    {
        const double a = __hiloint2double((int)((w >> 3 & 0x0FFFFFFFu) | 0x30000000u), (int)(w << 29));
        s = fma(a, a, s);
    }
};

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
    double s = 0.0, t = 0.0, u = 0.0, w = 0.0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        NormShare<T>::squares(raw[i].x, s, t);
        NormShare<T>::squares(raw[i].y, u, w);
        NormShare<T>::squares(raw[i].z, s, t);
        NormShare<T>::squares(raw[i].w, u, w);
    }
    const double sum = (s + t) + (u + w);
    if (sum >= 0x1p-436 && sum < 1.0) return sum * 0x1p256;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) any |= raw[i].x | raw[i].y | raw[i].z | raw[i].w;
    if ((any & NormShare<T>::MAGNITUDE) == 0) return 0.0;
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
// What every element of a step needs.  The corrections are folded in: with r = sqrt(inv_c2),
//   lr (inv_c1 m / (sqrt(inv_c2 v) + eps) + wd P) = rate (m / (sqrt(v) + eps / r) + decay P),  rate = lr inv_c1 / r,  decay = wd r / inv_c1.
struct Scalars { float rate, decay, eps, factor; uint32_t t_lo, t_hi; };

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
    int whole_grid;                      // 8 bits: blocks of threads for whole tiles; the tensors' ends have the others
    const float* factor;
    const float* lr_at;
    const long long* t_at;
    float b1, a1, b2, a2;                // a = 1 - b
    double lr, wd, eps, inv_c1, root;    // root = sqrt(inv_c2)
    double log_b1, log_b2;               // for the step count on the device
    int bias_correction;
    int fast;                            // 8 bits: eps is large enough for FLUSHED roots
    unsigned long long t;
    Scalars scalars;
    uint32_t keys[20];
};

__host__ __device__ inline Scalars scalars_of(double lr, double wd, double eps, double inv_c1, double root, unsigned long long t)
{
    Scalars s;
    s.rate = (float)(lr * inv_c1 / root);
    s.decay = (float)(wd * root / inv_c1);
    s.eps = (float)(eps / root);
    s.factor = 1.0f;
    s.t_lo = (uint32_t)t; s.t_hi = (uint32_t)(t >> 32);
    return s;
}

// By one thread of a block; the host's unless lr or the step count is on the device.
template <int CAP>
__device__ __forceinline__ Scalars read_scalars(const ListArgs<CAP>& a)
{
    Scalars s = a.scalars;
    if (a.lr_at || a.t_at) {
        const double lr = a.lr_at ? *a.lr_at : a.lr;
        double inv_c1 = a.inv_c1, root = a.root;
        unsigned long long t = a.t;
        if (a.t_at) {
            t = (unsigned long long)*a.t_at;
            if (a.bias_correction) {
                inv_c1 = -1.0 / expm1((double)(t + 1) * a.log_b1);
                root = sqrt(-1.0 / expm1((double)(t + 1) * a.log_b2));
            }
        }
        s = scalars_of(lr, a.wd, a.eps, inv_c1, root, t);
    }
    if (a.factor) s.factor = *a.factor;
    return s;
}

// Pairs of floats in one 64-bit register: one instruction for two elements.
__device__ __forceinline__ uint64_t pair2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
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
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Roots and quotients are rounded correctly where that is free (moments of 32 bits: 262 M in 844 us, 843 without).  The step of 8 bits is bound by
// instruction issue (262 M bfloat16: 614 us instead of 472) and takes them from the special-function unit, relative errors about 2^-23, beside
// codes of three bits.  FLUSHED drops what is below the normal range: a root that is off by 1.1e-19 at most, beside an eps of 1e-12 or more nothing;
// a smaller eps takes APPROXIMATE (three instructions more each).
enum : int { APPROXIMATE, FLUSHED, EXACT };
template <int HOW>
__device__ __forceinline__ float root_of(float x)
{
    float y;
    if constexpr (HOW == FLUSHED) asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    else asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int HOW>
__device__ __forceinline__ float inverse_of(float x)
{
    float y;
    if constexpr (HOW == FLUSHED) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    else asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// m, v and p of eight elements, one step on: m comes in as b1 m = scale * m[].  Every product and sum of m and v is rounded by itself, as a
// program of elementwise operations in fp32 rounds them: the same bits, so the same codes (fused: 2 instructions an element less, and one
// code in two million another one).  The sums are not in pairs: the compiler fuses a product and a sum of pairs although both say .rn.
struct Update {
    uint64_t factor, a1, b2, a2, eps, rate, decay;
    template <int CAP>
    __device__ __forceinline__ Update(const ListArgs<CAP>& a, const Scalars& s)
        : factor(pair2(s.factor, s.factor)), a1(pair2(a.a1, a.a1)), b2(pair2(a.b2, a.b2)), a2(pair2(a.a2, a.a2)),
          eps(pair2(s.eps, s.eps)), rate(pair2(-s.rate, -s.rate)), decay(pair2(s.decay, s.decay)) {}
    template <int HOW>
    __device__ __forceinline__ void apply(const float (&g)[8], float scale, float (&m)[8], float (&v)[8], float (&p)[8]) const
    {
        const uint64_t b1 = pair2(scale, scale);
#pragma unroll
        for (int x = 0; x < 8; x += 2) {
            const uint64_t gg = mul2(pair2(g[x], g[x + 1]), factor);
            float s0, s1, t0, t1;
            unpack2(mul2(pair2(m[x], m[x + 1]), b1), s0, s1);
            unpack2(mul2(gg, a1), t0, t1);
            m[x] = __fadd_rn(s0, t0);
            m[x + 1] = __fadd_rn(s1, t1);
            unpack2(mul2(pair2(v[x], v[x + 1]), b2), s0, s1);
            unpack2(mul2(mul2(gg, gg), a2), t0, t1);
            v[x] = __fadd_rn(s0, t0);
            v[x + 1] = __fadd_rn(s1, t1);
            const uint64_t mm = pair2(m[x], m[x + 1]);
            float d0, d1;
            const uint64_t pp = pair2(p[x], p[x + 1]);
            uint64_t quotient;
            if constexpr (HOW == EXACT) {
                unpack2(add2(pair2(__fsqrt_rn(v[x]), __fsqrt_rn(v[x + 1])), eps), d0, d1);
                quotient = pair2(__fdiv_rn(m[x], d0), __fdiv_rn(m[x + 1], d1));
            } else {
                unpack2(add2(pair2(root_of<HOW>(v[x]), root_of<HOW>(v[x + 1])), eps), d0, d1);
                quotient = mul2(mm, pair2(inverse_of<HOW>(d0), inverse_of<HOW>(d1)));
            }
            unpack2(fma2(rate, fma2(decay, pp, quotient), pp), p[x], p[x + 1]);
        }
    }
};

// Exponent byte of a block whose largest magnitude has these bits, for codes of TOP + 1 binades.
template <int TOP>
__device__ __forceinline__ int exponent_of(uint32_t largest)
{
    const int e = (int)((largest + 0xFFFFFu) >> 23) - TOP;
    return min(max(e, 0), 255 - TOP);
}

__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t selector)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(selector));
    return r;
}

// Largest of three, NaN if one is.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t largest_bits(const float (&x)[8])
{
    float r = max3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2]));
    r = max3(r, fabsf(x[3]), fabsf(x[4]));
    r = max3(r, fabsf(x[5]), fabsf(x[6]));
    return __float_as_uint(max3(r, fabsf(x[7]), fabsf(x[7])));
}

// Four integers cut to [0, 255], a byte each.
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d)
{
    uint32_t hi, r;
    asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(hi) : "r"(d), "r"(c), "r"(0));
    asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(b), "r"(a), "r"(hi));
    return r;
}
// The top bytes of four words.
__device__ __forceinline__ uint32_t top4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return permute(permute(a, b, 0x0073), permute(c, d, 0x0073), 0x5410);
}

// m's codes as floats for k = 112 (exponents -15 ... 0): times 2^(k - 112) they are the values, for every k but the lowest, whose first codes
// are subnormal, and the highest, whose last ones are infinity and NaN.
__device__ __forceinline__ float code_value(int b)
{
    const uint32_t c = b & 127;
    return __uint_as_float((c ? (c << 20) + (112u << 23) : 0u) | (uint32_t)(b & 128) << 24);
}

// Codes to values; m = scale * m[].
__device__ __forceinline__ void decode8(uint2 cm, uint2 cv, uint32_t k, const float* table, float& scale, float (&m)[8], float (&v)[8])
{
    const uint32_t km = k & 255u, kv = (k >> 8) << 23;
#pragma unroll
    for (int x = 0; x < 8; ++x)           // the code in bits 16 to 23
        v[x] = __uint_as_float(permute(x < 4 ? cv.x : cv.y, 0, 0x4044 | (x & 3) << 8) * 16 + kv);
    if (km - 1u < 239u) {
        scale = __uint_as_float((km + 15u) << 23);
#pragma unroll
        for (int x = 0; x < 8; ++x) m[x] = table[permute(x < 4 ? cm.x : cm.y, 0, 0x4440 | (x & 3))];
        return;
    }
    scale = 1.0f;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        // the code in bits 16 to 23, its sign in those above too
        uint32_t f = permute(x < 4 ? cm.x : cm.y, 0, 0x8044 | (x & 3) << 12 | (x & 3) << 8) * 16 & 0x87F00000u;
        if (f & 0x07F00000u) f += km << 23;
        m[x] = __uint_as_float(f);
    }
}

__device__ __forceinline__ void encode8(const float (&m)[8], const float (&v)[8], uint4 r4, uint2& cm, uint2& cv, uint32_t& k)
{
    const uint32_t top_m = __reduce_max_sync(0xFFFFFFFFu, largest_bits(m)), top_v = __reduce_max_sync(0xFFFFFFFFu, largest_bits(v));
    const int km = exponent_of<15>(top_m), kv = exponent_of<31>(top_v);
    uint32_t r[4] = { r4.x, r4.y, r4.z, r4.w };
    if (max(top_m, top_v) >= 0x7F800000u) r[0] = r[1] = r[2] = r[3] = 0;       // an infinity or NaN is not rounded on
    // Codes are bits 20 to 26 (m, its sign is bit 31) and 20 to 27 (v) of these, unless an element is below the lowest one.
    uint32_t em[8], ev[8], out_m = 0, out_v = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const uint32_t dither = permute(r[x >> 1], 0, x & 1 ? 0x4432 : 0x4410) * 16;
        em[x] = __float_as_uint(m[x]) + dither - ((uint32_t)km << 23);
        ev[x] = __float_as_uint(v[x]) + dither - ((uint32_t)kv << 23);
        out_m |= em[x];
        out_v |= ev[x];
    }
    k = (uint32_t)(km | kv << 8);
    if ((out_m & 0x78000000u) == 0 && out_v < 0x10000000u) {
        uint32_t bm[8], bv[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            bm[x] = (em[x] * 16 & 0x7FFFFFFFu) | (em[x] & 0x80000000u);
            bv[x] = ev[x] * 16;
        }
        cm = make_uint2(top4(bm[0], bm[1], bm[2], bm[3]), top4(bm[4], bm[5], bm[6], bm[7]));
        cv = make_uint2(top4(bv[0], bv[1], bv[2], bv[3]), top4(bv[4], bv[5], bv[6], bv[7]));
        return;
    }
    int cut[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) cut[x] = (int)(em[x] ^ (__float_as_uint(m[x]) & 0x80000000u)) >> 20;
    const uint32_t sign[2] = { top4(__float_as_uint(m[0]), __float_as_uint(m[1]), __float_as_uint(m[2]), __float_as_uint(m[3])),
                               top4(__float_as_uint(m[4]), __float_as_uint(m[5]), __float_as_uint(m[6]), __float_as_uint(m[7])) };
    cm.x = (pack4(cut[0], cut[1], cut[2], cut[3]) & 0x7F7F7F7Fu) | (sign[0] & 0x80808080u);
    cm.y = (pack4(cut[4], cut[5], cut[6], cut[7]) & 0x7F7F7F7Fu) | (sign[1] & 0x80808080u);
#pragma unroll
    for (int x = 0; x < 8; ++x) cut[x] = (int)ev[x] >> 20;
    cv = make_uint2(pack4(cut[0], cut[1], cut[2], cut[3]), pack4(cut[4], cut[5], cut[6], cut[7]));
}

// Loads run a tile ahead of the arithmetic, through a ring of blocks in shared memory that each warp has for itself: a warp waits for no
// other one, and its registers hold one block.  Copies are 512 contiguous bytes an instruction (with lanes 32 bytes apart every
// sector of fp32 was fetched twice: 1.4 times the time).
__device__ __forceinline__ void copy16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to), "l"(from) : "memory");
}
// A block of 256 elements to shared memory, from the lane's 16 bytes on.  fp32: a lane will read two pieces side by side; every other
// group of eight pieces is swapped in pairs, so that neither read hits a bank twice.
__device__ __forceinline__ void copy_block(uint32_t to, const __nv_bfloat16* from, int lane) { copy16(to + lane * 16, from); }
__device__ __forceinline__ void copy_block(uint32_t to, const float* from, int lane)
{
    const uint32_t at = to + (lane ^ (lane >> 3 & 1)) * 16;
    copy16(at, from);
    copy16(at + 512, from + 128);
}
__device__ __forceinline__ Raw8<__nv_bfloat16> read_block(const char* from, int lane, __nv_bfloat16)
{
    return Raw8<__nv_bfloat16>{ reinterpret_cast<const uint4*>(from)[lane] };
}
__device__ __forceinline__ Raw8<float> read_block(const char* from, int lane, float)
{
    const int at = 2 * lane, flip = lane >> 2 & 1;
    return Raw8<float>{ reinterpret_cast<const float4*>(from)[at ^ flip], reinterpret_cast<const float4*>(from)[(at + 1) ^ flip] };
}
// (a tensor's last elements: `count` of them, zeros behind)
__device__ __forceinline__ Raw8<float> guarded(const float* p, int count)
{
    float v[8];
    load8_guarded(p, count, v);
    return Raw8<float>{ make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]) };
}
__device__ __forceinline__ Raw8<__nv_bfloat16> guarded(const __nv_bfloat16* p, int count)
{
    float v[8];
    load8_guarded(p, count, v);
    return Raw8<__nv_bfloat16>{ make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])) };
}

// The tensor that a tile belongs to.
template <int CAP>
__device__ __forceinline__ int find_tensor(const ListArgs<CAP>& a, int tile)
{
    int at = 0, hi = a.n;
    while (hi - at > 1) {
        const int mid = (at + hi) >> 1;
        if (a.tile_begin[mid] <= tile) at = mid; else hi = mid;
    }
    return at;
}

// A tile is RING blocks of each warp, side by side: the warps' first blocks, their second ones, ...
template <typename PT, typename GT>
struct Stage {
    static constexpr int P = 0, G = P + AL_BLOCK * sizeof(PT), M = G + AL_BLOCK * sizeof(GT), V = M + AL_BLOCK, BYTES = V + AL_BLOCK;
    static constexpr int RING = 4, BLOCKS = RING * AL_WARPS, TILE = BLOCKS * AL_BLOCK, SMEM = BLOCKS * BYTES;
    static constexpr int FIT = 227 * 1024 / (SMEM + 2 * 1024), RESIDENT = FIT < 3 ? FIT : 3;
};

// 8 bits.  Bound by instruction issue with bfloat16 weights and gradients (50 an element, of which Philox 5, decoding 9, encoding 13; the
// issue limit at the copy rate is 55), by memory otherwise.  What that shaped:
//   * m's codes are looked up in shared memory (an add that must not happen for code 0 costs three instructions more);
//   * pairs of floats (fma.rn.f32x2) for the update;
//   * codes are cut out of four words at a time, clamped only where an element of a lane is below the lowest code;
//   * whole tiles and the tensors' ends are different blocks of threads: with both in one loop it took 5 instructions an element more;
//   * up to AL_WAVES times as many blocks as are resident: with one wave the slowest multiprocessor sets the time (529 us for 504);
//   * loads through registers instead: 613 us (too few bytes under way beside what the arithmetic holds).
// 262 M parameters: bfloat16 472 us, 5.6 TB/s; fp32 weights with bfloat16 gradients 550, all fp32 622 (at the copy rate 401, 561, 641), in twenty
// calls at 1965 MHz.  Bound by issue it goes with the clock: after seconds of it the board is at 1000 W and 1760 MHz, bfloat16 559 us.  With lr and the
// step count on the device bfloat16 takes 482 (every block works the scalars out), the others the same.
template <typename PT, typename GT, int CAP>
__global__ void __launch_bounds__(AL_THREADS, (Stage<PT, GT>::RESIDENT))
adamw8_kernel(const __grid_constant__ ListArgs<CAP> a)
{
    using S = Stage<PT, GT>;
    constexpr int RING = S::RING, STEP = AL_WARPS * AL_BLOCK;
    extern __shared__ __align__(16) char ring[];
    __shared__ Scalars shared;
    __shared__ float table[256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto prologue = [&] {
        if (threadIdx.x == 0) shared = read_scalars(a);
        table[threadIdx.x] = code_value((int)threadIdx.x);
        __syncthreads();
        return shared;
    };
    auto step = [&](const Scalars& s, const Update& update, const Raw8<PT>& rp, const Raw8<GT>& rg, int block, float (&p)[8], uint2& cm, uint2& cv, uint32_t& k) {
        float g[8], m[8], v[8], scale;
        unpack_raw8(rp, p);
        unpack_raw8(rg, g);
        decode8(cm, cv, k, table, scale, m, v);
        if (a.fast) update.template apply<FLUSHED>(g, scale * a.b1, m, v, p);
        else update.template apply<APPROXIMATE>(g, scale * a.b1, m, v, p);
        encode8(m, v, philox4x32_10_keys((uint32_t)block, (uint32_t)lane, s.t_lo, s.t_hi, a.keys), cm, cv, k);
    };
    if ((int)blockIdx.x >= a.whole_grid) {             // the end of a tensor, behind its last whole tile
        const int at = (int)blockIdx.x - a.whole_grid;
        const long long numel = a.numel[at], done = numel / S::TILE * S::TILE;
        if (done == numel) return;
        const Scalars s = prologue();
        if (!isfinite(s.factor)) return;
        const Update update(a, s);
#pragma unroll 1
        for (long long e = done + warp * AL_BLOCK; e < numel; e += STEP) {
            const int block = a.block_begin[at] + (int)(e / AL_BLOCK), count = (int)max(0ll, min(8ll, numel - e - lane * 8));
            const long long se = (long long)block * AL_BLOCK + lane * 8;
            PT* const P = static_cast<PT*>(a.p[at]) + e + lane * 8;
            const GT* const G = static_cast<const GT*>(a.g[at]) + e + lane * 8;
            const Raw8<PT> rp = count == 8 ? load_raw8_stream(P) : guarded(P, count);
            const Raw8<GT> rg = count == 8 ? load_raw8_stream(G) : guarded(G, count);
            uint2 cm = *reinterpret_cast<const uint2*>(a.m + se), cv = *reinterpret_cast<const uint2*>(a.v + se);
            uint32_t k = a.k[block];
            float p[8];
            step(s, update, rp, rg, block, p, cm, cv, k);
            if (count == 8) {
                store8(P, p);
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) if (x < count) store1(P + x, p[x]);
            }
            *reinterpret_cast<uint2*>(a.m + se) = cm;
            *reinterpret_cast<uint2*>(a.v + se) = cv;
            if (lane == 0) a.k[block] = (uint16_t)k;
        }
        return;
    }
    const char* const mine = ring + warp * (RING * S::BYTES);
    const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
    const int tiles = a.tile_begin[a.n];
    // The warp's first block of a tile: the lane's elements and codes of it, its number.
    struct Place { PT* p; const GT* g; char* m; char* v; int block; };
    auto find = [&](int tile) {
        const int at = find_tensor(a, tile), local = (tile - a.tile_begin[at]) * S::BLOCKS + warp, block = a.block_begin[at] + local;
        const long long e = (long long)local * AL_BLOCK + lane * 8, se = (long long)block * AL_BLOCK + lane * 8;
        return Place{ static_cast<PT*>(a.p[at]) + e, static_cast<const GT*>(a.g[at]) + e, a.m + se, a.v + se, block };
    };
    // Copies the warp's block i of a tile and closes a group.
    auto fetch = [&](const Place& w, bool there, int i) {
        if (there) {
            const uint32_t to = mine_at + i * S::BYTES;
            copy_block(to + S::P, w.p + i * STEP + lane * (16 / (int)sizeof(PT) - 8), lane);
            copy_block(to + S::G, w.g + i * STEP + lane * (16 / (int)sizeof(GT) - 8), lane);
            copy8(to + S::M + lane * 8, w.m + i * STEP);
            copy8(to + S::V + lane * 8, w.v + i * STEP);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // The exponents of the warp's blocks, one a lane.
    auto exponents = [&](const Place& w) { return lane < RING ? a.k[w.block + lane * AL_WARPS] : (uint16_t)0; };
    int tile = blockIdx.x;
    Place now = find(tile);
#pragma unroll
    for (int i = 0; i < RING; ++i) fetch(now, true, i);
    uint32_t k = exponents(now);
    const Scalars s = prologue();
    if (!isfinite(s.factor)) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    const Update update(a, s);
    for (; tile < tiles; tile += a.whole_grid) {
        const bool more = tile + a.whole_grid < tiles;
        const Place next = more ? find(tile + a.whole_grid) : now;
        const uint32_t next_k = exponents(next);
#pragma unroll 1
        for (int i = 0; i < RING; ++i) {
            asm volatile("cp.async.wait_group %0;" :: "n"(RING - 1) : "memory");
            __syncwarp();                              // what the other lanes copied is there as well
            const char* const from = mine + i * S::BYTES;
            const Raw8<PT> rp = read_block(from + S::P, lane, PT());
            const Raw8<GT> rg = read_block(from + S::G, lane, GT());
            uint2 cm = reinterpret_cast<const uint2*>(from + S::M)[lane], cv = reinterpret_cast<const uint2*>(from + S::V)[lane];
            uint32_t kk = __shfl_sync(0xFFFFFFFFu, k, i);
            __syncwarp();                              // every lane has read: the next tile's block takes its place
            fetch(next, more, i);
            float p[8];
            step(s, update, rp, rg, now.block + i * AL_WARPS, p, cm, cv, kk);
            store8(now.p + i * STEP, p);
            __stcs(reinterpret_cast<uint2*>(now.m + i * STEP), cm);
            __stcs(reinterpret_cast<uint2*>(now.v + i * STEP), cv);
            if (lane == i) k = kk;
        }
        if (lane < RING) a.k[now.block + lane * AL_WARPS] = (uint16_t)k;
        now = next;
        k = next_k;
    }
}

// Moments of 32 bits: nothing but the traffic.  A block of threads has one tile, so that fast and slow multiprocessors share the work as
// they can (blocks that stay and loop: 906 us instead of 842).  262 M parameters: bfloat16 844 us, 6.8 TB/s; fp32 weights with bfloat16
// gradients 1000, all fp32 1069 (at the copy rate 882, 1042, 1122); with lr and the step count on the device the same.
template <typename PT, typename GT, int CAP>
__global__ void __launch_bounds__(AL_THREADS, 4)
adamw32_kernel(const __grid_constant__ ListArgs<CAP> a)
{
    __shared__ Scalars shared;
    if (threadIdx.x == 0) shared = read_scalars(a);
    __syncthreads();
    const Scalars s = shared;
    if (!isfinite(s.factor)) return;
    const Update update(a, s);
    const int at = find_tensor(a, blockIdx.x);
    const long long first = (long long)(blockIdx.x - a.tile_begin[at]) * AL_TILE32;
    const long long left = a.numel[at] - first;
    PT* const P = static_cast<PT*>(a.p[at]) + first;
    const GT* const G = static_cast<const GT*>(a.g[at]) + first;
    float* const M = reinterpret_cast<float*>(a.m) + (long long)a.block_begin[at] * AL_BLOCK + first;
    float* const V = reinterpret_cast<float*>(a.v) + (long long)a.block_begin[at] * AL_BLOCK + first;
#pragma unroll 1
    for (int e = threadIdx.x * 8; e < AL_TILE32; e += AL_THREADS * 8) {
        const int count = (int)max(0ll, min(8ll, left - e));
        if (count == 0) break;
        float g[8], p[8], m[8], v[8];
        if (count == 8) { load8_stream(P + e, p); load8_stream(G + e, g); load8_stream(M + e, m); load8_stream(V + e, v); }
        else { load8_guarded(P + e, count, p); load8_guarded(G + e, count, g); load8_guarded(M + e, count, m); load8_guarded(V + e, count, v); }
        update.template apply<EXACT>(g, a.b1, m, v, p);
        if (count == 8) { store8(P + e, p); store8(M + e, m); store8(V + e, v); }
        else {
#pragma unroll
            for (int x = 0; x < 8; ++x) if (x < count) { store1(P + e + x, p[x]); M[e + x] = m[x]; V[e + x] = v[x]; }
        }
    }
}

// Values of 8-bit moments, sixteen elements a thread, a block for each 4096 (262 M: 242 us, 6.5 TB/s; blocks that loop: 327 us).
__global__ void __launch_bounds__(AL_THREADS)
adamw_moments_kernel(const uint4* __restrict__ cm, const uint4* __restrict__ cv, const uint16_t* __restrict__ ks, long long n,
                     uint4* __restrict__ m, uint4* __restrict__ v)
{
    const long long i = (long long)blockIdx.x * AL_THREADS + threadIdx.x;
    if (i < n) {
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

template <typename PT, typename GT, int CAP>
cudaError_t list_launch(ListArgs<CAP>& a, bool q8, int sms, cudaStream_t stream)
{
    using S = Stage<PT, GT>;
    int64_t tiles = 0;
    bool ends = false;
    for (int k = 0; k < a.n; ++k) {
        a.tile_begin[k] = (int)tiles;
        tiles += q8 ? a.numel[k] / S::TILE : (a.numel[k] + AL_TILE32 - 1) / AL_TILE32;
        ends |= a.numel[k] % S::TILE != 0;
    }
    a.tile_begin[a.n] = (int)tiles;
    if (!q8) {
        adamw32_kernel<PT, GT, CAP><<<(unsigned)tiles, AL_THREADS, 0, stream>>>(a);
        return cudaGetLastError();
    }
    static std::atomic<unsigned long long> allowed{ 0 };
    const cudaError_t e = allow_shared(adamw8_kernel<PT, GT, CAP>, S::SMEM, allowed);
    if (e != cudaSuccess) return e;
    const int64_t most = (int64_t)S::RESIDENT * sms * AL_WAVES;
    a.whole_grid = (int)(tiles < most ? tiles : most);
    adamw8_kernel<PT, GT, CAP><<<(unsigned)(a.whole_grid + (ends ? a.n : 0)), AL_THREADS, S::SMEM, stream>>>(a);
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
    int64_t block = 0;
    a.n = 0;
    for (int32_t i = 0; i <= c.n; ++i) {
        if ((i == c.n || a.n == CAP) && a.n > 0) {
            const bool pb = dp == APOLLO_DT_BF16, gb = dg == APOLLO_DT_BF16;
            const cudaError_t e = pb ? (gb ? list_launch<__nv_bfloat16, __nv_bfloat16>(a, c.q8, c.sms, c.stream) : list_launch<__nv_bfloat16, float>(a, c.q8, c.sms, c.stream))
                                     : (gb ? list_launch<float, __nv_bfloat16>(a, c.q8, c.sms, c.stream) : list_launch<float, float>(a, c.q8, c.sms, c.stream));
            if (e != cudaSuccess) return APOLLO_ERR_CUDA;
            a.n = 0;
        }
        if (i == c.n) break;
        const int64_t blocks = (c.numel[i] + AL_BLOCK - 1) / AL_BLOCK;
        if (c.G[i] && blocks > 0 && c.dtype_P[i] == dp && c.dtype_G[i] == dg) {
            a.p[a.n] = c.P[i]; a.g[a.n] = c.G[i]; a.numel[a.n] = c.numel[i];
            a.block_begin[a.n] = (int)block;
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
    a.lr = lr; a.wd = wd; a.eps = cfg->eps;
    a.b1 = (float)cfg->beta1; a.a1 = (float)(1.0 - cfg->beta1); a.b2 = (float)cfg->beta2; a.a2 = (float)(1.0 - cfg->beta2);
    a.bias_correction = cfg->bias_correction;
    a.fast = cfg->eps >= 1e-12;
    a.log_b1 = std::log(cfg->beta1); a.log_b2 = std::log(cfg->beta2);      // (-inf for 0: expm1 is -1, c = 1)
    a.inv_c1 = a.root = 1.0;
    if (cfg->bias_correction) {
        a.inv_c1 = -1.0 / std::expm1(((double)t + 1) * a.log_b1);
        a.root = std::sqrt(-1.0 / std::expm1(((double)t + 1) * a.log_b2));
    }
    a.t = (unsigned long long)t;
    a.scalars = scalars_of(lr, wd, cfg->eps, a.inv_c1, a.root, a.t);
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
    const char* m = static_cast<const char*>(d_state);
    const char* v = m + (size_t)n_blocks * AL_BLOCK;
    const int64_t vectors = n_blocks * (AL_BLOCK / 16);
    adamw_moments_kernel<<<(unsigned)((vectors + AL_THREADS - 1) / AL_THREADS), AL_THREADS, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        reinterpret_cast<const uint4*>(m), reinterpret_cast<const uint4*>(v), reinterpret_cast<const uint16_t*>(v + (size_t)n_blocks * AL_BLOCK),
        vectors, static_cast<uint4*>(d_M), static_cast<uint4*>(d_V));
    return cudaGetLastError() == cudaSuccess ? APOLLO_OK : APOLLO_ERR_CUDA;
}
