// An AdamW step of all replicas, with or without the elastic exchange, and the norms that clip their gradients.
//
// Per worker i and parameter j (see include/easgd.h for the definition):
//   g = clip G;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   W <- W - eta (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay W) - eta rho (W - c);   Wc <- c + eta rho sum_i (W_i - c)
// Every operand is read once and every result written once.  Bound: HBM.
#include "logits.h"

namespace easgd {

typedef float Four __attribute__((ext_vector_type(4)));

struct AdamwArgs {
    float *W;
    void *M, *S;
    float *M_scale, *S_scale;          // [P][blocks]: of the moments in 8 bits
    const void *G;
    float *Wc;
    int P;
    size_t N, ld, blocks;
    const long long *ends;             // [tensors]: where they end
    const float *rates, *decays;
    int tensors;
    const float *clip;
    float eta;
    const float *eta_at;
    float rho, beta1, beta2, eps, decay;
    long long step;
    const long long *step_at;
    unsigned seed;
};

// ---- numbers of a step ------------------------------------------------------------------------------------------------
struct StepNumbers {
    float eta, alpha, beta1, beta2, rest1, rest2, eps, decay;
    float by1, by2;                    // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
    unsigned step;                     // its lower 32 bits
    __device__ __forceinline__ explicit StepNumbers(const AdamwArgs &a)
    {
        const long long t = a.step_at ? max(a.step_at[0], 1ll) : a.step;
        eta = a.eta_at ? a.eta_at[0] : a.eta;
        alpha = eta * a.rho;
        beta1 = a.beta1;
        beta2 = a.beta2;
        rest1 = 1.f - beta1;
        rest2 = 1.f - beta2;
        eps = a.eps;
        decay = a.decay;
        by1 = (float)(1.0 / (1.0 - power((double)beta1, t)));
        by2 = (float)(1.0 / sqrt(1.0 - power((double)beta2, t)));
        step = (unsigned)t;
    }
    // x^t for 0 <= x < 1 by squaring
    __device__ static __forceinline__ double power(double x, long long t)
    {
        double p = 1.0;
        for (; t > 0 && p > 0.0; t >>= 1, x *= x)
            if (t & 1) p *= x;
        return p;
    }
};

// A parameter's rate and decay: those of its tensor, or the call's behind the last one's end.
struct TensorWalk {
    const AdamwArgs &a;
    int at;                            // the first tensor that ends behind the parameter
    __device__ __forceinline__ TensorWalk(const AdamwArgs &a, size_t j) : a(a), at(0)
    {
        int n = a.tensors;             // binary search: ends ascend
        while (n > 0) {
            const int half = n >> 1;
            if ((size_t)a.ends[at + half] <= j) {
                at += half + 1;
                n -= half + 1;
            } else n = half;
        }
    }
    __device__ __forceinline__ void to(size_t j)
    {
        while (at < a.tensors && (size_t)a.ends[at] <= j) ++at;
    }
    __device__ __forceinline__ size_t end() const { return at < a.tensors ? (size_t)a.ends[at] : ~(size_t)0; }
    __device__ __forceinline__ float rate() const { return at < a.tensors ? a.rates[at] : 1.f; }
    __device__ __forceinline__ float decay() const { return at < a.tensors ? a.decays[at] : a.decay; }
};

// What multiplies m / (sqrt(v) + eps) and w of a lane's four parameters in a block of 256; nearly always one tensor has the whole block.
__device__ __forceinline__ bool in_one_tensor(const TensorWalk &tensor, size_t block) { return tensor.end() >= block * 256 + 256; }
struct Pace {
    float rate[4], decay[4];
    __device__ __forceinline__ Pace(float r, float d)
    {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            rate[q] = r;
            decay[q] = d;
        }
    }
    __device__ __forceinline__ Pace(const AdamwArgs &a, const StepNumbers &n, size_t block, size_t j)
    {
        TensorWalk tensor(a, block * 256);
        const bool one = in_one_tensor(tensor, block);  // uniform
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (!one) tensor.to(j + q);
            const float eta = n.eta * tensor.rate();
            rate[q] = eta * n.by1;
            decay[q] = eta * tensor.decay();
        }
    }
};
// The same for the blocks of a tile: two numbers a block, and eight a lane, kept in LDS, where a tensor ends inside one.
template <int GROUPS> struct TilePace {
    float rate[GROUPS], decay[GROUPS];
    bool one[GROUPS];
    Four (*lanes)[2][256];             // [GROUPS]: rates and decays, a thread's own
    __device__ __forceinline__ explicit TilePace(Four (*lanes)[2][256]) : lanes(lanes) {}
    __device__ __forceinline__ void set(const AdamwArgs &a, const StepNumbers &n, int q, size_t block, size_t j)
    {
        const TensorWalk tensor(a, block * 256);
        one[q] = in_one_tensor(tensor, block);
        const float eta = n.eta * tensor.rate();
        rate[q] = eta * n.by1;
        decay[q] = eta * tensor.decay();
        if (!one[q]) {                                  // uniform for the wavefront
            const Pace pace(a, n, block, j);
            lanes[q][0][threadIdx.x] = (Four){pace.rate[0], pace.rate[1], pace.rate[2], pace.rate[3]};
            lanes[q][1][threadIdx.x] = (Four){pace.decay[0], pace.decay[1], pace.decay[2], pace.decay[3]};
        }
    }
    __device__ __forceinline__ Pace of(int q) const
    {
        Pace pace(rate[q], decay[q]);
        if (!one[q]) {
            const Four r = lanes[q][0][threadIdx.x], d = lanes[q][1][threadIdx.x];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pace.rate[e] = r[e];
                pace.decay[e] = d[e];
            }
        }
        return pace;
    }
};

// ---- the rule of one parameter -------------------------------------------------------------------------------------------
// The moments' arithmetic decides stored codes of 8 bits, so it is pinned: every operation is rounded on its own.
__device__ __forceinline__ void adamw_moments(float &m, float &v, float g, const StepNumbers &n)
{
#pragma clang fp contract(off)
    m = m * n.beta1 + g * n.rest1;
    v = v * n.beta2 + (g * n.rest2) * g;
}
// What four parameters move by: eta (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay w).  The hardware's root and reciprocal are right to
// one unit; it takes subnormal numbers for 0, so roots of what is below 2^-64 are taken of 2^64 times it.  eps is at least 1e-30: the
// reciprocal is of a normal number.  The quotient comes first and the rate then, as in the formula: rate times reciprocal may be above what 32 bits
// hold (a large rate over a small eps) where the quotient is 0.
__device__ __forceinline__ void adamw_move(const float (&w)[4], const float (&m)[4], const float (&v)[4], const Pace &pace, const StepNumbers &n, float (&move)[4])
{
    float root[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) root[q] = __builtin_amdgcn_sqrtf(v[q]);
    if (__any(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < 0x1p-64f)) {         // uniform
#pragma unroll
        for (int q = 0; q < 4; ++q) root[q] = v[q] < 0x1p-64f ? __builtin_amdgcn_sqrtf(v[q] * 0x1p64f) * 0x1p-32f : root[q];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float d = fmaf(root[q], n.by2, n.eps);
        move[q] = fmaf(pace.decay[q], w[q], m[q] * __builtin_amdgcn_rcpf(d) * pace.rate[q]);
    }
}

// ---- moments in 8 bits -----------------------------------------------------------------------------------------------------
// 256 consecutive parameters of a replica share a power of two per moment: the largest |m| of them lands in [2^7, 2^8) of e4m3,
// the largest v in [2^14, 2^15) of e5m2, and a number x of 2^-e m (2^-e v) becomes one of its two neighbours, at random, with its
// distance from the other one as probability: exact on average (but for a v above 0 that is less than the type's smallest number: it is raised to that, never
// 0), where rounding to the nearest would never let v move (b2 = 0.999 changes it by 0.1 % a step, half a step of the type is 12 %).  Multiplied by 2^-120 (2^-112) the type's exponents are those of fp32,
// subnormal numbers included, so 16 random bits are added below the last kept one, and what is behind it is cut off.
// The random bits of parameter j = 4 g + 2 w + h of worker i in step t are half h of mix(g ^ key(i, t, w)).
__device__ __forceinline__ unsigned mix(unsigned x)
{
    x = (x ^ x >> 16) * 0x6C8E9CF5u;
    x = (x ^ x >> 15) * 0x2F5D7A4Bu;
    return x ^ x >> 16;
}
__device__ __forceinline__ unsigned dither_key(unsigned seed, unsigned worker, unsigned step, unsigned word)
{
    return mix(mix(seed + worker * 0x9E3779B1u) + step * 0x85157AF5u + word * 0x632BE5ABu);
}
// bits: of the type's fraction; top: exponent of the largest number's place
template <int BITS, int TOP> struct EightBits {
    static constexpr int UNIT = BITS == 2 ? -112 : -120;
    unsigned scale;                    // biased exponent of the block's power of two
    bool there;                        // neither infinite nor NaN in the block
    __device__ __forceinline__ explicit EightBits(unsigned most)        // the largest magnitude of the block, as bits
    {
        there = most < 0x7f800000u;
        scale = (unsigned)max((int)(most >> 23) - TOP, 1);
    }
    // (codes under the scale NaN say nothing)
    __device__ __forceinline__ float stored() const { return there ? __uint_as_float(scale << 23) : NAN; }
    // fp32 bits whose upper part, from bit 23 - BITS on, is the code (of a magnitude), random: 20 bits
    __device__ __forceinline__ unsigned code(float x, unsigned random) const
    {
        return __float_as_uint(__builtin_amdgcn_ldexpf(x, 127 + UNIT - (int)scale)) + (random << (3 - BITS));
    }
};
using MomentM = EightBits<3, 7>;
using MomentS = EightBits<2, 14>;

// Codes of four moments in a word, from the sums that code() gave.
__device__ __forceinline__ unsigned pack_m(const unsigned (&y)[4])
{
    unsigned t[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = (y[q] << 4 & 0x7fffffffu) | (y[q] & 0x80000000u);          // the code in the upper byte
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[3], t[2], 0x0c0c0703u), __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0703u), 0x05040100u);
}
__device__ __forceinline__ unsigned pack_s(const unsigned (&y)[4], const float (&v)[4])
{
    unsigned t[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = max(y[q] >> 21, min(__float_as_uint(v[q]), 1u));           // what is above 0 stays above 0
    return (t[3] << 8 | t[2]) << 16 | (t[1] << 8 | t[0]);
}

// the largest magnitude's bits over a wavefront: within rows of 16 lanes by data-parallel moves, then the four rows as scalars
__device__ __forceinline__ unsigned wave_max_bits(unsigned v)
{
    auto with = [&](unsigned other) { v = max(v, other); };
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));        // lane ^ 1
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));        // lane ^ 2
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));       // 8 lanes mirrored
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));       // 16 lanes mirrored
    const unsigned a = (unsigned)__builtin_amdgcn_readlane((int)v, 0), b = (unsigned)__builtin_amdgcn_readlane((int)v, 16);
    const unsigned c = (unsigned)__builtin_amdgcn_readlane((int)v, 32), d = (unsigned)__builtin_amdgcn_readlane((int)v, 48);
    return max(max(a, b), max(c, d));
}

// ---- four consecutive parameters of a lane ------------------------------------------------------------------------------------
// How they are accessed: at once past the caches (what is read once and written once), at once, or element by element with a look at the
// row's end (the last 256 parameters).  The hardware's wide accesses need the element's alignment only, so rows of any stride take them.
enum { ACCESS_STREAM, ACCESS_WIDE, ACCESS_EACH };
template <typename T, int ACCESS> __device__ __forceinline__ void load_four(const T *p, size_t j, size_t N, T (&x)[4])
{
    typedef T Vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if constexpr (ACCESS == ACCESS_EACH) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = j + i < N ? p[j + i] : (T)0;
    } else {
        const Vec *at = reinterpret_cast<const Vec *>(p + j);
        Vec v;
        if constexpr (ACCESS == ACCESS_STREAM) v = __builtin_nontemporal_load(at);
        else v = *at;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
}
template <typename T, int ACCESS> __device__ __forceinline__ void store_four(T *p, size_t j, size_t N, const T (&x)[4])
{
    typedef T Vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if constexpr (ACCESS == ACCESS_EACH) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i < N) p[j + i] = x[i];
    } else {
        const Vec v = {x[0], x[1], x[2], x[3]};
        Vec *at = reinterpret_cast<Vec *>(p + j);
        if constexpr (ACCESS == ACCESS_STREAM) __builtin_nontemporal_store(v, at);
        else *at = v;
    }
}

// four codes in a word
typedef unsigned Codes __attribute__((aligned(1)));
template <int ACCESS> __device__ __forceinline__ unsigned load_codes(const unsigned char *p, size_t j, size_t N)
{
    if constexpr (ACCESS == ACCESS_EACH) {
        unsigned char c[4];
        load_four<unsigned char, ACCESS>(p, j, N, c);
        return (unsigned)c[3] << 24 | (unsigned)c[2] << 16 | (unsigned)c[1] << 8 | c[0];
    } else if constexpr (ACCESS == ACCESS_STREAM) return __builtin_nontemporal_load(reinterpret_cast<const Codes *>(p + j));
    else return *reinterpret_cast<const Codes *>(p + j);
}
template <int ACCESS> __device__ __forceinline__ void store_codes(unsigned char *p, size_t j, size_t N, unsigned codes)
{
    if constexpr (ACCESS == ACCESS_EACH) {
        const unsigned char c[4] = {(unsigned char)codes, (unsigned char)(codes >> 8), (unsigned char)(codes >> 16), (unsigned char)(codes >> 24)};
        store_four<unsigned char, ACCESS>(p, j, N, c);
    } else if constexpr (ACCESS == ACCESS_STREAM) __builtin_nontemporal_store((Codes)codes, reinterpret_cast<Codes *>(p + j));
    else *reinterpret_cast<Codes *>(p + j) = codes;
}

// A worker's share of 256 parameters, four of them a lane's, between loads and stores.
template <int GT, bool EIGHT, int ACCESS> struct Worker {
    using Grad = typename LogitType<GT>::Stored;
    float w[4], m[4], v[4];
    Grad g[4];
    unsigned mc, vc;                   // four codes each
    float ms, vs;                      // scales, the same for all lanes
    __device__ __forceinline__ void load_moments(const AdamwArgs &a, int i, size_t j)
    {
        const size_t row = (size_t)i * a.ld;
        load_four<Grad, ACCESS>((const Grad *)a.G + row, j, a.N, g);
        if constexpr (EIGHT) {
            mc = load_codes<ACCESS>((const unsigned char *)a.M + row, j, a.N);
            vc = load_codes<ACCESS>((const unsigned char *)a.S + row, j, a.N);
            const size_t block = (size_t)i * a.blocks + __builtin_amdgcn_readfirstlane((unsigned)(j >> 8));
            ms = a.M_scale[block];
            vs = a.S_scale[block];
        } else {
            load_four<float, ACCESS>((const float *)a.M + row, j, a.N, m);
            load_four<float, ACCESS>((const float *)a.S + row, j, a.N, v);
        }
    }
    __device__ __forceinline__ void load_parameters(const AdamwArgs &a, int i, size_t j) { load_four<float, ACCESS>(a.W + (size_t)i * a.ld, j, a.N, w); }
    // new moments, and what the parameters move by
    __device__ __forceinline__ void step(const AdamwArgs &a, int i, size_t j, float clip, const Pace &pace, const StepNumbers &n, float (&move)[4])
    {
        if constexpr (EIGHT) {
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                const auto pm = q ? __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, false);
                const auto pv = q ? __builtin_amdgcn_cvt_pk_f32_bf8((int)vc, true) : __builtin_amdgcn_cvt_pk_f32_bf8((int)vc, false);
                m[q] = pm[0] * ms;
                m[q + 1] = pm[1] * ms;
                v[q] = pv[0] * vs;
                v[q + 1] = pv[1] * vs;
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) adamw_moments(m[q], v[q], clip * LogitType<GT>::widen(g[q]), n);
        adamw_move(w, m, v, pace, n, move);
        if constexpr (EIGHT) {
            unsigned most_m = 0, most_v = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool in = ACCESS != ACCESS_EACH || j + q < a.N;
                most_m = max(most_m, in ? __float_as_uint(m[q]) << 1 : 0u);
                most_v = max(most_v, in ? __float_as_uint(v[q]) : 0u);           // v >= 0, or NaN of either sign
            }
            const MomentM em(wave_max_bits(most_m) >> 1);
            const MomentS es(wave_max_bits(most_v));
            ms = em.stored();
            vs = es.stored();
            unsigned ym[4], yv[4];
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                const unsigned h = mix((unsigned)(j >> 2) ^ dither_key(a.seed, i, n.step, q >> 1));
                const unsigned low = ((h & 0xffffu) << 4) + 8u, high = (h >> 16 << 4) + 8u;
                ym[q] = em.code(m[q], low);
                ym[q + 1] = em.code(m[q + 1], high);
                yv[q] = es.code(v[q], low);
                yv[q + 1] = es.code(v[q + 1], high);
            }
            mc = pack_m(ym);
            vc = pack_s(yv, v);
        }
    }
    __device__ __forceinline__ void store_moments(const AdamwArgs &a, int i, size_t j)
    {
        const size_t row = (size_t)i * a.ld;
        if constexpr (EIGHT) {
            store_codes<ACCESS>((unsigned char *)a.M + row, j, a.N, mc);
            store_codes<ACCESS>((unsigned char *)a.S + row, j, a.N, vc);
            const size_t block = (size_t)i * a.blocks + __builtin_amdgcn_readfirstlane((unsigned)(j >> 8));
            if ((threadIdx.x & 63) == 0) {
                a.M_scale[block] = ms;
                a.S_scale[block] = vs;
            }
        } else {
            store_four<float, ACCESS>((float *)a.M + row, j, a.N, m);
            store_four<float, ACCESS>((float *)a.S + row, j, a.N, v);
        }
    }
    __device__ __forceinline__ void store_parameters(const AdamwArgs &a, int i, size_t j) { store_four<float, ACCESS>(a.W + (size_t)i * a.ld, j, a.N, w); }
};

// One block of 256 parameters by a wavefront, workers [i0, i1).
template <int GT, bool EIGHT, bool CENTER, int ACCESS>
__device__ __forceinline__ void adamw_block(const AdamwArgs &a, const StepNumbers &n, size_t block, int i0, int i1)
{
    const size_t j = block * 256 + (size_t)(threadIdx.x & 63) * 4;
    const Pace pace(a, n, block, j);
    float c[4] = {}, sum[4] = {};
    if constexpr (CENTER) load_four<float, ACCESS == ACCESS_EACH ? ACCESS_EACH : ACCESS_WIDE>(a.Wc, j, a.N, c);
    for (int i = i0; i < i1; ++i) {                     // ascending: fixed order of the sum
        const float clip = a.clip ? a.clip[i] : 1.f;
        if (!CENTER && clip == 0.f) continue;           // it sits the step out
        Worker<GT, EIGHT, ACCESS> worker;
        float move[4] = {};
        worker.load_parameters(a, i, j);
        if (clip != 0.f) {
            worker.load_moments(a, i, j);
            worker.step(a, i, j, clip, pace, n, move);
            worker.store_moments(a, i, j);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (CENTER) {
                const float d = worker.w[q] - c[q];
                sum[q] += d;
                move[q] = fmaf(n.alpha, d, move[q]);
            }
            worker.w[q] -= move[q];
        }
        worker.store_parameters(a, i, j);
    }
    if constexpr (CENTER) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c[q] = fmaf(n.alpha, sum[q], c[q]);
        store_four<float, ACCESS == ACCESS_EACH ? ACCESS_EACH : ACCESS_WIDE>(a.Wc, j, a.N, c);
    }
}

// ---- no center: a wavefront per 256 parameters of a worker (blockIdx.y) -------------------------------------------------------------------
template <int GT, bool EIGHT, int ACCESS>
__global__ __launch_bounds__(256) void adamw_own_kernel(AdamwArgs a)
{
    const size_t block = (size_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (block >= a.blocks) return;                      // wavefronts of a block have nothing in common
    const StepNumbers n(a);
    const int i = (int)blockIdx.y;
    if (block < a.N / 256) adamw_block<GT, EIGHT, false, ACCESS>(a, n, block, i, i + 1);
    else adamw_block<GT, EIGHT, false, ACCESS_EACH>(a, n, block, i, i + 1);
}

// ---- a center and few parameters: 256 of them a block, whose wavefronts take the workers in turn ------------------------------------------
// What the workers are apart from the center meets in LDS, SPLIT_ROOM workers at a time, and is added in ascending order: the same sums as
// worker by worker.  Four wavefronts a block (eight, or two, are slower), whose requests for two workers are under way at a time (one with moments in 8 bits):
// 16 x 1.86 M, bf16 gradients, one worker sitting out, 142 us = 5.3 TB/s, all working 151 = 5.2 (a wavefront for all workers 174 us, room for 32 workers 163, which leaves a compute unit five blocks in the
// place of eight).
static constexpr int SPLIT_ROOM = 16;
template <int GT, bool EIGHT, int ACCESS, int WAVES>
__device__ __forceinline__ void adamw_split_block(const AdamwArgs &a, const StepNumbers &n, size_t block, Four (&apart)[SPLIT_ROOM][64])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t j = block * 256 + (size_t)lane * 4;
    const Pace pace(a, n, block, j);
    constexpr int SPLIT_AHEAD = EIGHT ? 1 : 2;
    constexpr int CENTER_ACCESS = ACCESS == ACCESS_EACH ? ACCESS_EACH : ACCESS_WIDE;
    float c[4];
    load_four<float, CENTER_ACCESS>(a.Wc, j, a.N, c);
    Four sum = {0.f, 0.f, 0.f, 0.f};
    for (int first = 0; first < a.P; first += SPLIT_ROOM) {
        const int end = min(first + SPLIT_ROOM, a.P);
        for (int i0 = first + wave; i0 < end; i0 += SPLIT_AHEAD * WAVES) {
            Worker<GT, EIGHT, ACCESS> worker[SPLIT_AHEAD];
            float clip[SPLIT_AHEAD];
#pragma unroll
            for (int u = 0; u < SPLIT_AHEAD; ++u) {
                const int i = i0 + u * WAVES;
                if (i >= end) break;
                clip[u] = a.clip ? a.clip[i] : 1.f;
                if (clip[u] != 0.f) worker[u].load_moments(a, i, j);
                worker[u].load_parameters(a, i, j);
            }
#pragma unroll
            for (int u = 0; u < SPLIT_AHEAD; ++u) {
                const int i = i0 + u * WAVES;
                if (i >= end) break;
                float move[4] = {};
                if (clip[u] != 0.f) {
                    worker[u].step(a, i, j, clip[u], pace, n, move);
                    worker[u].store_moments(a, i, j);
                }
                Four d;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    d[q] = worker[u].w[q] - c[q];
                    worker[u].w[q] -= fmaf(n.alpha, d[q], move[q]);
                }
                apart[i - first][lane] = d;
                worker[u].store_parameters(a, i, j);
            }
        }
        __syncthreads();
        if (wave == 0)
            for (int i = first; i < end; ++i) sum += apart[i - first][lane];
        __syncthreads();
    }
    if (wave != 0) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) c[q] = fmaf(n.alpha, sum[q], c[q]);
    store_four<float, CENTER_ACCESS>(a.Wc, j, a.N, c);
}
template <int GT, bool EIGHT, int ACCESS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void adamw_split_kernel(AdamwArgs a)
{
    __shared__ Four apart[SPLIT_ROOM][64];
    const StepNumbers n(a);
    if (blockIdx.x < a.N / 256) adamw_split_block<GT, EIGHT, ACCESS, WAVES>(a, n, blockIdx.x, apart);      // uniform
    else adamw_split_block<GT, EIGHT, ACCESS_EACH, WAVES>(a, n, blockIdx.x, apart);
}

// ---- many parameters: GROUPS blocks of 256 a wavefront, all requests of a worker under way at once -------------------------------------
// Which blocks those are is the TileMap of the other streaming updates: the dies interleave.  Bound: HBM.  8 x 61 M fp32, call after call on the same replicas:
// moments in 32 bits 2 180 us = 6.3 TB/s, with the center 2 217 = 6.4; in 8 bits 1 322 us = 5.9 TB/s, with the center 1 360 = 6.1 (1 410 where other
// calls come between), the vector ALUs 71 % busy (some 59 instructions a parameter: decoding, the rule, two maxima over 256 parameters, random bits, codes;
// 1 660 us for the first such kernel).
// With moments in 32 bits two wavefronts a vector ALU and no more: fewer, longer bursts of requests stream faster (without / with the center: 2 180 / 2 217 us,
// with three 2 243 / 2 264, with four 2 245 / 2 489).
template <int GT, bool EIGHT, bool CENTER, bool NT, int GROUPS, bool DIES>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(EIGHT ? 1 : 2, EIGHT ? 8 : 2))) void adamw_tile_kernel(AdamwArgs a)
{
    typedef TileMap<GROUPS, DIES> Map;
    constexpr int ACCESS = NT ? ACCESS_STREAM : ACCESS_WIDE;
    const size_t full = a.N / 256;
    const StepNumbers n(a);
    const size_t first = Map::first(blockIdx.x, threadIdx.x), lead = Map::first(blockIdx.x, threadIdx.x & ~63u) >> 6;       // in groups of four; the wavefront's first block
    const size_t b0 = (size_t)__builtin_amdgcn_readfirstlane((unsigned)lead);
    constexpr size_t STEP = Map::STRIDE >> 6;
    if (b0 + (GROUPS - 1) * STEP >= full) {             // uniform for the wavefront: at the row's end
#pragma unroll 1
        for (int q = 0; q < GROUPS; ++q) {
            const size_t block = b0 + q * STEP;
            if (block < full) adamw_block<GT, EIGHT, CENTER, ACCESS_WIDE>(a, n, block, 0, a.P);
            else if (block < a.blocks) adamw_block<GT, EIGHT, CENTER, ACCESS_EACH>(a, n, block, 0, a.P);
        }
        return;
    }
    size_t j[GROUPS];
    float c[GROUPS][4], sum[GROUPS][4] = {};
    __shared__ Four lanes[GROUPS][2][256];
    TilePace<GROUPS> pace(lanes);
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
        j[q] = (first + q * Map::STRIDE) * 4;
        pace.set(a, n, q, b0 + q * STEP, j[q]);
        if constexpr (CENTER) load_four<float, ACCESS_WIDE>(a.Wc, j[q], a.N, c[q]);
    }
    for (int i = 0; i < a.P; ++i) {                     // ascending: fixed order of the sum
        const float clip = a.clip ? a.clip[i] : 1.f;
        if (!CENTER && clip == 0.f) continue;           // it sits the step out
        Worker<GT, EIGHT, ACCESS> worker[GROUPS];
        if (clip != 0.f) {
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) worker[q].load_moments(a, i, j[q]);
        }
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) worker[q].load_parameters(a, i, j[q]);
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            float move[4] = {};
            if (clip != 0.f) worker[q].step(a, i, j[q], clip, pace.of(q), n, move);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (CENTER) {
                    const float d = worker[q].w[e] - c[q][e];
                    sum[q][e] += d;
                    move[e] = fmaf(n.alpha, d, move[e]);
                }
                worker[q].w[e] -= move[e];
            }
        }
        if (clip != 0.f) {
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) worker[q].store_moments(a, i, j[q]);
        }
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) worker[q].store_parameters(a, i, j[q]);
    }
    if constexpr (CENTER) {
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
#pragma unroll
            for (int e = 0; e < 4; ++e) c[q][e] = fmaf(n.alpha, sum[q][e], c[q][e]);
            store_four<float, ACCESS_WIDE>(a.Wc, j[q], a.N, c[q]);
        }
    }
}

// ---- norms -------------------------------------------------------------------------------------------------------------------------
// Squares are added in 64 bits: no gradient is too large or too small for them, and the order of addition is fixed.  Bound: HBM.  8 x 61 M fp32
// 286 us = 6.8 TB/s (element by element 536); 16 x 1.86 M bf16 13 us, two launches.
struct NormArgs {
    const void *G;
    int P;
    size_t N, ld;
    float max_norm, *norm, *clip;
    int parts;
    double *partial;                   // [P][parts]
};
__device__ __forceinline__ void write_norm(const NormArgs &a, int i, double sum)
{
    const double norm = sqrt(sum);
    const float stored = (float)norm;
    a.norm[i] = stored;
    if (a.clip) a.clip[i] = !(stored < INFINITY) ? 0.f : norm <= (double)a.max_norm ? 1.f : (float)((double)a.max_norm / norm);
}
// A row is cut into tiles of BLOCK * DEEP slots of 128 bits on the 16-byte grid; part p of it has tiles p, p + parts, ...: the chip reads
// one window of memory at a time.  The elements in front of the first slot and behind the last one are part 0's.
template <int GT, int BLOCK, int DEEP>
__global__ __launch_bounds__(BLOCK) void norm_parts_kernel(NormArgs a)
{
    using Type = LogitType<GT>;
    using Stored = typename Type::Stored;
    constexpr int VEC = Type::VEC;
    typedef unsigned Words __attribute__((ext_vector_type(4)));
    __shared__ double scratch[BLOCK / 64];
    const int i = blockIdx.y;
    const Stored *row = (const Stored *)a.G + (size_t)i * a.ld;
    const size_t skip = (size_t)((16u - ((uintptr_t)row & 15u)) & 15u) / sizeof(Stored), head = skip < a.N ? skip : a.N, slots = (a.N - head) / VEC;
    const Words *at = reinterpret_cast<const Words *>(row + head);
    double sum[2] = {0.0, 0.0};
    auto add = [&](const Words &w) {
        float x[VEC];
        Type::unpack(make_uint4(w[0], w[1], w[2], w[3]), x);
#pragma unroll
        for (int q = 0; q < VEC; ++q) sum[q & 1] = fma((double)x[q], (double)x[q], sum[q & 1]);
    };
    constexpr size_t TILE = (size_t)BLOCK * DEEP;
    for (size_t t = blockIdx.x; t * TILE < slots; t += a.parts) {
        const size_t s = t * TILE + threadIdx.x;
        Words w[DEEP];
        if ((t + 1) * TILE <= slots) {                  // uniform
#pragma unroll
            for (int q = 0; q < DEEP; ++q) w[q] = __builtin_nontemporal_load(at + s + q * BLOCK);
#pragma unroll
            for (int q = 0; q < DEEP; ++q) add(w[q]);
        } else {
#pragma unroll
            for (int q = 0; q < DEEP; ++q)
                if (s + q * BLOCK < slots) add(at[s + q * BLOCK]);
        }
    }
    if (blockIdx.x == 0) {
        const size_t tail = head + slots * VEC;
        auto one = [&](size_t j) {
            const double x = (double)Type::widen(row[j]);
            sum[0] = fma(x, x, sum[0]);
        };
        if (threadIdx.x < head) one(threadIdx.x);
        if (tail + threadIdx.x < a.N) one(tail + threadIdx.x);
    }
    const double all = block_sum<BLOCK>(sum[0] + sum[1], scratch);
    if (threadIdx.x != 0) return;
    if (a.parts == 1) write_norm(a, i, all);
    else a.partial[(size_t)i * a.parts + blockIdx.x] = all;
}
__global__ __launch_bounds__(64) void norm_join_kernel(NormArgs a)
{
    const int i = blockIdx.x;
    double sum = 0.0;
    for (int p = threadIdx.x; p < a.parts; p += 64) sum += a.partial[(size_t)i * a.parts + p];
    sum = wave_sum(sum);
    if (threadIdx.x == 0) write_norm(a, i, sum);
}

// ---- host --------------------------------------------------------------------------------------------------------------------------
static constexpr size_t MOST_N = (size_t)1 << 34;       // groups of four have numbers of 32 bits
static int check_replicas(const char *name, const void *G, int dtype, int P, size_t N, size_t ld)
{
    if (!G) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (dtype != EASGD_F32 && dtype != EASGD_BF16 && dtype != EASGD_F16) return fail(EASGD_EINVAL, "%s: unknown element type %d", name, dtype);
    if (P < 1) return fail(EASGD_EINVAL, "%s: P must be >= 1, got %d", name, P);
    if (N == 0) return fail(EASGD_EINVAL, "%s: N must be >= 1", name);
    if (ld < N) return fail(EASGD_EINVAL, "%s: ld (%zu) < N (%zu)", name, ld, N);
    if (P > 65535) return fail(EASGD_ERANGE, "%s: more than 65535 workers", name);
    if (N > MOST_N || ld > ((size_t)1 << 60) / (size_t)P) return fail(EASGD_ERANGE, "%s: N or P * ld too large", name);
    if (!aligned_to(G, dtype_bytes(dtype))) return fail(EASGD_EINVAL, "%s: G must be aligned to its elements (%zu bytes)", name, dtype_bytes(dtype));
    return EASGD_OK;
}

// Rows of up to NORM_ONE bytes take one block of 1024 threads each and one launch.
static constexpr int NORM_BLOCK = 256, NORM_DEEP = 8, NORM_BLOCKS = 2048;
static constexpr size_t NORM_ONE = (size_t)256 << 10, NORM_TILE = (size_t)NORM_BLOCK * NORM_DEEP * 16;
static int norm_parts(int P, size_t bytes)
{
    if (bytes <= NORM_ONE) return 1;
    const size_t most = (bytes + NORM_TILE - 1) / NORM_TILE, want = (size_t)((NORM_BLOCKS + P - 1) / P);
    return (int)(want < most ? want : most);
}

// Tiles where every compute unit gets 64 blocks of 256 and more; with 16, 8 x 1 M takes 40 us against 35 for a wavefront a worker and block.
// Tiles of 8 x 61 M, us (1 / 2 / 4 blocks of 256 a wavefront): moments in 32 bits 2428 / 2237 / 2180, with the center 2671 / 2261 / 2217; in 8 bits 1420 / 1322 /
// 1301, with the center 1415 / 1360 / 1471: these need more wavefronts under way, whose arithmetic hides behind each other's loads.
template <int GT, bool EIGHT, bool CENTER> static void launch_adamw(const AdamwArgs &a, hipStream_t s)
{
    constexpr int GROUPS = EIGHT ? 2 : 4;
    const bool stream = update_nontemporal((size_t)a.P * a.N * (8 + (GT == EASGD_F32 ? 4 : 2) + (EIGHT ? 4 : 16)));
    if (a.blocks >= (size_t)64 * num_cus()) {
        const dim3 grid((unsigned)TileMap<GROUPS, true>::tiles(a.blocks * 64));
        // codes of rows at other alignments share lines between neighbouring pieces: through the caches and one die after the other (30 x 6 M packed 680 us,
        // interleaved past the caches 781; with moments in 32 bits there is no difference: 8 x 30 M 1 385 to 1 438 us)
        const bool apart = EIGHT && (a.ld % 4 != 0 || !aligned_to(a.M, 4) || !aligned_to(a.S, 4));
        if (apart) EASGD_LAUNCH((adamw_tile_kernel<GT, EIGHT, CENTER, false, GROUPS, !EIGHT>), dim3((unsigned)TileMap<GROUPS, !EIGHT>::tiles(a.blocks * 64)), dim3(256), 0, s, a);
        else if (stream) EASGD_LAUNCH((adamw_tile_kernel<GT, EIGHT, CENTER, true, GROUPS, true>), grid, dim3(256), 0, s, a);
        else EASGD_LAUNCH((adamw_tile_kernel<GT, EIGHT, CENTER, false, GROUPS, true>), grid, dim3(256), 0, s, a);
    } else if constexpr (CENTER) {
        const dim3 grid((unsigned)a.blocks);
        if (stream) EASGD_LAUNCH((adamw_split_kernel<GT, EIGHT, ACCESS_STREAM, 4>), grid, dim3(256), 0, s, a);
        else EASGD_LAUNCH((adamw_split_kernel<GT, EIGHT, ACCESS_WIDE, 4>), grid, dim3(256), 0, s, a);
    } else {
        const dim3 grid((unsigned)((a.blocks + 3) / 4), (unsigned)a.P);
        if (stream) EASGD_LAUNCH((adamw_own_kernel<GT, EIGHT, ACCESS_STREAM>), grid, dim3(256), 0, s, a);
        else EASGD_LAUNCH((adamw_own_kernel<GT, EIGHT, ACCESS_WIDE>), grid, dim3(256), 0, s, a);
    }
}

template <bool EIGHT> static int adamw(const char *name, AdamwArgs a, int dtype, void *stream)
{
    if (!a.W || !a.M || !a.S || (EIGHT && (!a.M_scale || !a.S_scale))) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (int rc = check_replicas(name, a.G, dtype, a.P, a.N, a.ld)) return rc;
    if (!aligned_to(a.W, 4) || !aligned_to(a.Wc, 4) || !aligned_to(a.M_scale, 4) || !aligned_to(a.S_scale, 4) || !aligned_to(a.clip, 4) || !aligned_to(a.eta_at, 4) ||
        (!EIGHT && (!aligned_to(a.M, 4) || !aligned_to(a.S, 4))))
        return fail(EASGD_EINVAL, "%s: fp32 pointers must be 4-byte aligned", name);
    if (a.tensors < 0 || (a.tensors > 0 && (!a.ends || !a.rates || !a.decays))) return fail(EASGD_EINVAL, "%s: %d tensors need ends, rates and decays", name, a.tensors);
    if (!aligned_to(a.ends, 8) || !aligned_to(a.rates, 4) || !aligned_to(a.decays, 4) || !aligned_to(a.step_at, 8))
        return fail(EASGD_EINVAL, "%s: ends, step_at must be 8-byte, rates, decays 4-byte aligned", name);
    if (!(a.beta1 >= 0.f && a.beta1 < 1.f) || !(a.beta2 >= 0.f && a.beta2 < 1.f))
        return fail(EASGD_EINVAL, "%s: beta1 and beta2 must be in [0, 1), got %g and %g", name, (double)a.beta1, (double)a.beta2);
    if (!(a.eps >= 1e-30f && a.eps <= 1e30f)) return fail(EASGD_EINVAL, "%s: eps must be in [1e-30, 1e30], got %g", name, (double)a.eps);
    if (!std::isfinite(a.eta) || !std::isfinite(a.rho) || !std::isfinite(a.decay)) return fail(EASGD_EINVAL, "%s: eta, rho and decay must be finite", name);
    if (!a.Wc && a.rho != 0.f) return fail(EASGD_EINVAL, "%s: rho = %g needs a center", name, (double)a.rho);
    if (!a.step_at && a.step < 1) return fail(EASGD_EINVAL, "%s: step must be >= 1, got %lld", name, a.step);
    clear_error();
    a.blocks = (a.N + 255) / 256;
    if (a.tensors == 0) a.ends = nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto gt) {
        constexpr int GT = decltype(gt)::value;
        if (a.Wc) launch_adamw<GT, EIGHT, true>(a, s);
        else launch_adamw<GT, EIGHT, false>(a, s);
    });
    return check_launch(name);
}

}  // namespace easgd

extern "C" {

size_t easgd_grad_norms_workspace_bytes(int P, size_t N)
{
    using namespace easgd;
    if (P < 1 || N == 0 || N > MOST_N) return 0;
    const int parts = norm_parts(P, N * 4);             // fp32 rows have the most parts
    return parts == 1 ? 0 : ((size_t)P * parts * sizeof(double) + 255) / 256 * 256;
}

int easgd_grad_norms(const void *G, int dtype, int P, size_t N, size_t ld, float max_norm, float *norm, float *clip,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_grad_norms";
    if (int rc = check_replicas(name, G, dtype, P, N, ld)) return rc;
    if (!norm) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(norm, 4) || !aligned_to(clip, 4)) return fail(EASGD_EINVAL, "%s: norm, clip must be 4-byte aligned", name);
    if (!(max_norm > 0.f)) return fail(EASGD_EINVAL, "%s: max_norm must be above 0, got %g", name, (double)max_norm);
    if (int rc = check_workspace(name, workspace, workspace_bytes, easgd_grad_norms_workspace_bytes(P, N))) return rc;
    clear_error();
    const int parts = norm_parts(P, N * dtype_bytes(dtype));
    const NormArgs a = {G, P, N, ld, max_norm, norm, clip, parts, static_cast<double *>(workspace)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto gt) {
        constexpr int GT = decltype(gt)::value;
        if (parts == 1) EASGD_LAUNCH((norm_parts_kernel<GT, 1024, 4>), dim3(1, (unsigned)P), dim3(1024), 0, s, a);
        else EASGD_LAUNCH((norm_parts_kernel<GT, NORM_BLOCK, NORM_DEEP>), dim3((unsigned)parts, (unsigned)P), dim3(NORM_BLOCK), 0, s, a);
    });
    if (parts > 1) EASGD_LAUNCH(norm_join_kernel, dim3((unsigned)P), dim3(64), 0, s, a);
    return check_launch(name);
}

int adamw_round(float *W, float *M, float *S, const void *G, int dtype, float *Wc, int P, size_t N, size_t ld,
                const int64_t *ends, const float *rates, const float *decays, int tensors, const float *clip,
                float eta, const float *eta_at, float rho, float beta1, float beta2, float eps, float decay,
                int64_t step, const int64_t *step_at, void *stream)
{
    easgd::AdamwArgs a = {W, M, S, nullptr, nullptr, G, Wc, P, N, ld, 0, reinterpret_cast<const long long *>(ends), rates, decays, tensors, clip,
                          eta, eta_at, rho, beta1, beta2, eps, decay, (long long)step, reinterpret_cast<const long long *>(step_at), 0u};
    return easgd::adamw<false>("adamw_round", a, dtype, stream);
}

int adamw_round_8bit(float *W, uint8_t *M, uint8_t *S, float *M_scale, float *S_scale, const void *G, int dtype, float *Wc, int P, size_t N, size_t ld,
                     const int64_t *ends, const float *rates, const float *decays, int tensors, const float *clip,
                     float eta, const float *eta_at, float rho, float beta1, float beta2, float eps, float decay,
                     int64_t step, const int64_t *step_at, uint32_t seed, void *stream)
{
    easgd::AdamwArgs a = {W, M, S, M_scale, S_scale, G, Wc, P, N, ld, 0, reinterpret_cast<const long long *>(ends), rates, decays, tensors, clip,
                          eta, eta_at, rho, beta1, beta2, eps, decay, (long long)step, reinterpret_cast<const long long *>(step_at), seed};
    return easgd::adamw<true>("adamw_round_8bit", a, dtype, stream);
}

}  // extern "C"
