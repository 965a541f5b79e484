// An AdamW step of all replicas, with or without the elastic exchange, and the norms that clip their gradients.
//
// Per worker i and parameter j (see include/easgd.h for the definition):
//   g = clip G;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   W <- W - eta (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay W) - eta rho (W - c);   Wc <- c + eta rho sum_i (W_i - c)
// Every operand is read once and every result written once.  Bound: HBM.
#include "logits.h"

namespace easgd {

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

// ---- the rule of one parameter -------------------------------------------------------------------------------------------
// The moments' arithmetic decides stored codes of 8 bits, so it is pinned: every operation is rounded on its own.
__device__ __forceinline__ void adamw_moments(float &m, float &v, float g, const StepNumbers &n)
{
#pragma clang fp contract(off)
    m = m * n.beta1 + g * n.rest1;
    v = v * n.beta2 + (g * n.rest2) * g;
}
// What a parameter moves by: eta (m' / (sqrt(v') + eps) + decay w)
__device__ __forceinline__ float adamw_move(float w, float m, float v, float eta, float decay, const StepNumbers &n)
{
    const float d = fmaf(sqrtf(v), n.by2, n.eps);
    return eta * fmaf(decay, w, m * n.by1 / d);
}

// ---- moments in 8 bits -----------------------------------------------------------------------------------------------------
// 256 consecutive parameters of a replica share a power of two per moment: the largest |m| of them lands in [2^7, 2^8) of e4m3,
// the largest v in [2^14, 2^15) of e5m2, and a number x of 2^-e m (2^-e v) becomes one of its two neighbours, at random, with its
// distance from the other one as probability: exact on average, where rounding to the nearest would never let v move (b2 = 0.999
// changes it by 0.1 % a step, half a step of the type is 12 %).  Multiplied by 2^-120 (2^-112) the type's exponents are those of fp32,
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
    static constexpr float UNIT = BITS == 2 ? 0x1p-112f : 0x1p-120f;
    unsigned scale;                    // biased exponent of the block's power of two
    bool there;                        // neither infinite nor NaN in the block
    __device__ __forceinline__ explicit EightBits(unsigned most)        // the largest magnitude of the block, as bits
    {
        there = most < 0x7f800000u;
        scale = (unsigned)max((int)(most >> 23) - TOP, 1);
    }
    __device__ __forceinline__ float stored() const { return there ? __uint_as_float(scale << 23) : NAN; }
    __device__ __forceinline__ unsigned code(float magnitude, unsigned dither) const
    {
#pragma clang fp contract(off)
        const float y = magnitude * __uint_as_float((254u - scale) << 23) * UNIT;
        return there ? (__float_as_uint(y) + (dither << (7 - BITS)) + (1u << (6 - BITS))) >> (23 - BITS) : 0u;
    }
};
using MomentM = EightBits<3, 7>;
using MomentS = EightBits<2, 14>;

__device__ __forceinline__ unsigned wave_max_bits(unsigned v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, o));
    return v;
}

// ---- four consecutive parameters ----------------------------------------------------------------------------------------------
typedef float Four __attribute__((ext_vector_type(4)));
// WIDE: all of a row's fours are aligned to their size, and read and stored at once
template <typename T, bool WIDE> __device__ __forceinline__ void load_four(const T *p, size_t j, size_t N, T (&x)[4])
{
    typedef T Vec __attribute__((ext_vector_type(4)));
    if (WIDE && j + 4 <= N) {
        const Vec v = *reinterpret_cast<const Vec *>(p + j);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = j + i < N ? p[j + i] : (T)0;
    }
}
template <typename T, bool WIDE> __device__ __forceinline__ void store_four(T *p, size_t j, size_t N, const T (&x)[4])
{
    typedef T Vec __attribute__((ext_vector_type(4)));
    if (WIDE && j + 4 <= N) {
        const Vec v = {x[0], x[1], x[2], x[3]};
        *reinterpret_cast<Vec *>(p + j) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i < N) p[j + i] = x[i];
    }
}

// ---- a wavefront per 256 parameters, worker by worker ------------------------------------------------------------------------------
template <int GT, bool EIGHT, bool CENTER, bool WIDE>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a)
{
    using Grad = typename LogitType<GT>::Stored;
    const size_t block = (size_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (block >= a.blocks) return;                      // wavefronts of a block have nothing in common
    const int lane = threadIdx.x & 63;
    const size_t j = block * 256 + (size_t)lane * 4;
    const StepNumbers n(a);
    float rate[4], decay[4];
    TensorWalk tensor(a, block * 256);
    if (tensor.end() >= block * 256 + 256) {            // uniform: one tensor for all
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            rate[q] = n.eta * tensor.rate();
            decay[q] = tensor.decay();
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            tensor.to(j + q);
            rate[q] = n.eta * tensor.rate();
            decay[q] = tensor.decay();
        }
    }
    float c[4] = {}, sum[4] = {};
    if constexpr (CENTER) load_four<float, WIDE>(a.Wc, j, a.N, c);
    for (int i = 0; i < a.P; ++i) {                     // ascending: fixed order of the sum
        const size_t row = (size_t)i * a.ld;
        const float clip = a.clip ? a.clip[i] : 1.f;
        float w[4], step[4] = {};
        load_four<float, WIDE>(a.W + row, j, a.N, w);
        if (clip != 0.f) {
            float m[4], v[4];
            Grad gs[4];
            load_four<Grad, WIDE>((const Grad *)a.G + row, j, a.N, gs);
            unsigned char mc[4], vc[4];
            float *const Ms = EIGHT ? a.M_scale + (size_t)i * a.blocks + block : nullptr, *const Ss = EIGHT ? a.S_scale + (size_t)i * a.blocks + block : nullptr;
            if constexpr (EIGHT) {
                load_four<unsigned char, WIDE>((const unsigned char *)a.M + row, j, a.N, mc);
                load_four<unsigned char, WIDE>((const unsigned char *)a.S + row, j, a.N, vc);
                const float ms = *Ms, vs = *Ss;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    m[q] = __builtin_amdgcn_cvt_f32_fp8((int)mc[q], 0) * ms;
                    v[q] = __builtin_amdgcn_cvt_f32_bf8((int)vc[q], 0) * vs;
                }
            } else {
                load_four<float, WIDE>((const float *)a.M + row, j, a.N, m);
                load_four<float, WIDE>((const float *)a.S + row, j, a.N, v);
            }
            unsigned most_m = 0, most_v = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                adamw_moments(m[q], v[q], clip * LogitType<GT>::widen(gs[q]), n);
                step[q] = adamw_move(w[q], m[q], v[q], rate[q], decay[q], n);
                if (j + q < a.N) {
                    most_m = max(most_m, __float_as_uint(m[q]) & 0x7fffffffu);
                    most_v = max(most_v, __float_as_uint(v[q]) & 0x7fffffffu);
                }
            }
            if constexpr (EIGHT) {
                const MomentM em(wave_max_bits(most_m));
                const MomentS es(wave_max_bits(most_v));
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const unsigned h = mix((unsigned)(j >> 2) ^ dither_key(a.seed, i, n.step, q >> 1)), dither = q & 1 ? h >> 16 : h & 0xffffu;
                    mc[q] = (unsigned char)(em.code(fabsf(m[q]), dither) | (m[q] < 0.f ? 0x80u : 0u));
                    vc[q] = (unsigned char)max(es.code(v[q], dither), v[q] > 0.f && es.there ? 1u : 0u);
                }
                store_four<unsigned char, WIDE>((unsigned char *)a.M + row, j, a.N, mc);
                store_four<unsigned char, WIDE>((unsigned char *)a.S + row, j, a.N, vc);
                if (lane == 0) {
                    *Ms = em.stored();
                    *Ss = es.stored();
                }
            } else {
                store_four<float, WIDE>((float *)a.M + row, j, a.N, m);
                store_four<float, WIDE>((float *)a.S + row, j, a.N, v);
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (CENTER) {
                const float d = w[q] - c[q];
                sum[q] += d;
                step[q] = fmaf(n.alpha, d, step[q]);
            }
            w[q] -= step[q];
        }
        store_four<float, WIDE>(a.W + row, j, a.N, w);
    }
    if constexpr (CENTER) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c[q] = fmaf(n.alpha, sum[q], c[q]);
        store_four<float, WIDE>(a.Wc, j, a.N, c);
    }
}

// ---- norms -------------------------------------------------------------------------------------------------------------------------
// Squares are added in 64 bits: no gradient is too large or too small for them, and the order of addition is fixed.
struct NormArgs {
    const void *G;
    int P;
    size_t N, ld;
    float max_norm, *norm, *clip;
    int parts;
    size_t part;                       // elements of a part of a row
    double *partial;                   // [P][parts]
};
__device__ __forceinline__ void write_norm(const NormArgs &a, int i, double sum)
{
    const double norm = sqrt(sum);
    const float stored = (float)norm;
    a.norm[i] = stored;
    if (a.clip) a.clip[i] = !(stored < INFINITY) ? 0.f : norm <= (double)a.max_norm ? 1.f : (float)((double)a.max_norm / norm);
}
template <int GT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_parts_kernel(NormArgs a)
{
    __shared__ double scratch[BLOCK / 64];
    const int i = blockIdx.y;
    const auto *g = (const typename LogitType<GT>::Stored *)a.G + (size_t)i * a.ld;
    const size_t j0 = (size_t)blockIdx.x * a.part, j1 = min(j0 + a.part, a.N);
    double sum = 0.0;
    for (size_t j = j0 + threadIdx.x; j < j1; j += BLOCK) {
        const double x = (double)LogitType<GT>::widen(g[j]);
        sum = fma(x, x, sum);
    }
    sum = block_sum<BLOCK>(sum, scratch);
    if (threadIdx.x != 0) return;
    if (a.parts == 1) write_norm(a, i, sum);
    else a.partial[(size_t)i * a.parts + blockIdx.x] = sum;
}
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_join_kernel(NormArgs a)
{
    __shared__ double scratch[BLOCK / 64];
    const int i = blockIdx.x;
    double sum = 0.0;
    for (int p = threadIdx.x; p < a.parts; p += BLOCK) sum += a.partial[(size_t)i * a.parts + p];
    sum = block_sum<BLOCK>(sum, scratch);
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
    if (N > MOST_N || ld > ((size_t)1 << 60) / (size_t)P) return fail(EASGD_ERANGE, "%s: N or P * ld too large", name);
    if (!aligned_to(G, dtype_bytes(dtype))) return fail(EASGD_EINVAL, "%s: G must be aligned to its elements (%zu bytes)", name, dtype_bytes(dtype));
    return EASGD_OK;
}

static constexpr int NORM_BLOCK = 256;
static constexpr size_t NORM_PART = 8192;
static int norm_parts(int P, size_t N)
{
    const size_t most = (N + NORM_PART - 1) / NORM_PART, want = (4096 + P - 1) / P;
    return (int)(want < most ? want : most);
}

template <int GT, bool EIGHT, bool WIDE> static void launch_adamw(const AdamwArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.blocks + 3) / 4));
    if (a.Wc) EASGD_LAUNCH((adamw_kernel<GT, EIGHT, true, WIDE>), grid, dim3(256), 0, s, a);
    else EASGD_LAUNCH((adamw_kernel<GT, EIGHT, false, WIDE>), grid, dim3(256), 0, s, a);
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
    if (!(a.eps > 0.f) || std::isinf(a.eps)) return fail(EASGD_EINVAL, "%s: eps must be finite and above 0, got %g", name, (double)a.eps);
    if (!std::isfinite(a.eta) || !std::isfinite(a.rho) || !std::isfinite(a.decay)) return fail(EASGD_EINVAL, "%s: eta, rho and decay must be finite", name);
    if (!a.Wc && a.rho != 0.f) return fail(EASGD_EINVAL, "%s: rho = %g needs a center", name, (double)a.rho);
    if (!a.step_at && a.step < 1) return fail(EASGD_EINVAL, "%s: step must be >= 1, got %lld", name, a.step);
    clear_error();
    a.blocks = (a.N + 255) / 256;
    if (a.tensors == 0) a.ends = nullptr;
    const size_t size = dtype_bytes(dtype);
    const bool wide = a.ld % 4 == 0 && aligned16(a.W) && aligned16(a.Wc) && aligned_to(a.G, 4 * size) && aligned_to(a.M, EIGHT ? 4 : 16) && aligned_to(a.S, EIGHT ? 4 : 16);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto gt) {
        constexpr int GT = decltype(gt)::value;
        if (wide) launch_adamw<GT, EIGHT, true>(a, s);
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
    const int parts = norm_parts(P, N);
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
    if (P > 65535) return fail(EASGD_ERANGE, "%s: more than 65535 workers", name);
    if (int rc = check_workspace(name, workspace, workspace_bytes, easgd_grad_norms_workspace_bytes(P, N))) return rc;
    clear_error();
    const int parts = norm_parts(P, N);
    const NormArgs a = {G, P, N, ld, max_norm, norm, clip, parts, (N + parts - 1) / parts, static_cast<double *>(workspace)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto gt) {
        EASGD_LAUNCH((norm_parts_kernel<decltype(gt)::value, NORM_BLOCK>), dim3((unsigned)parts, (unsigned)P), dim3(NORM_BLOCK), 0, s, a);
    });
    if (parts > 1) EASGD_LAUNCH((norm_join_kernel<NORM_BLOCK>), dim3((unsigned)P), dim3(NORM_BLOCK), 0, s, a);
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
