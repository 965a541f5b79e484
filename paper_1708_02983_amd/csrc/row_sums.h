// Sums of exponentials over a row of logits, at a temperature T (e_j) and, for the cross-entropy of a label, at 1 (h_j).
#pragma once
#include "logits.h"

namespace easgd {

// Where h_j comes from: nobody asks for it, or T is 1 and it is e_j; T is 2 and it is e_j^2 (a multiplication in the place of an
// exponential); an exponential of its own.
enum { HARD_PLAIN = 0, HARD_SQUARE = 1, HARD_EXP = 2 };

__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

struct Scales {
    float c, c1;              // log2(e) / T, and log2(e) where a cross-entropy asks for it
    __device__ __forceinline__ explicit Scales(float temperature, bool hard = false) : c((float)(LOG2E / (double)temperature)), c1(hard ? (float)LOG2E : c) {}
};

// Exponentials relative to a logit `ref`: 2^((x - ref) c) in one fused multiply-add and one exponential, as 2^(x c - rc) with
// rc = ref * c rounded once for all; what that rounding takes from every exponent alike, `lost`, is known exactly and goes
// into the row's factors.  That holds as long as `lost` is small, at most half a unit for |ref| c < 2^24.  Beyond:
//   * where even the type's next value is more than 2^8 units of the exponent away (2^-24 of ref for fp32, 2^-12 for fp16, more for
//     bfloat16), every other logit's exponential is 0 or infinite at any such scale, and a power of two, which multiplies exactly, does;
//   * between the two (fp32 logits from 2^24 T to 2^32 T, and some mixed temperatures) the difference comes first and is scaled then: an
//     instruction more a logit.  c is NaN there, so that the loops that do not know of it (one comparison a slot) find their sum to
//     be no number and look closer.
template <int VEC> struct Reference {
    float ref, c, c1, rc, rc1, lost, lost1;
    __device__ __forceinline__ Reference(const Scales &q) : ref(-INFINITY), c(q.c), c1(q.c1), rc(0.f), rc1(0.f), lost(0.f), lost1(0.f) {}
    __device__ __forceinline__ Reference(float r, const Scales &q) { set(r, q); }
    __device__ __forceinline__ void set(float r, const Scales &q)
    {
        constexpr float APART = VEC == 4 ? 0x1p32f : 0x1p20f;
        const float most = fabsf(r) * fmaxf(q.c, q.c1), least = fabsf(r) * fminf(q.c, q.c1);
        ref = r;
        c = q.c;
        c1 = q.c1;
        if (least >= APART) c = c1 = __uint_as_float((294u - (__float_as_uint(r) >> 23 & 255u)) << 23);      // |r| c in [2^40, 2^41)
        else if (most >= 0x1p24f) c = c1 = NAN;
        rc = r * c;
        rc1 = r * c1;
        lost = by_difference() ? 0.f : fmaf(r, c, -rc);               // the exponents are this much too large
        lost1 = by_difference() ? 0.f : fmaf(r, c1, -rc1);
    }
    __device__ __forceinline__ bool by_difference() const { return isnan(c); }
    __device__ __forceinline__ float soft(float x) const { return exp2_fast(fmaf(x, c, -rc)); }
    __device__ __forceinline__ float hard(float x) const { return exp2_fast(fmaf(x, c1, -rc1)); }
};

// Running sums of a thread, relative to a reference that its wavefront shares: the largest logit of the first slots that
// hold any, moved only when a slot's exponentials sum up to more than 2^24 (sums of 2^20 such terms are far from fp32's end),
// so that the loop over a row needs neither a maximum nor a rescaling, only a comparison per 128 bits.
//
// The sum outside the teacher's places is 0 if and only if every logit there is masked: where its terms are all below fp32, OUTSIDE_TINY
// stands for them.
static constexpr float OUTSIDE_TINY = 0x1p-100f;
template <int VEC, bool TAIL, int HARD> struct RowSums {
    const Scales &q;
    Reference<VEC> at;
    float st = 0.f, s1 = 0.f, so = 0.f;
    bool some = false;        // a logit above -inf outside the teacher's places: noted where nothing else tells of it
    bool settled = false;     // uniform: some lane has one, or a sum above 0

    __device__ __forceinline__ RowSums(const Scales &q) : q(q), at(q) {}
    // Whole wavefronts call it (lanes without a slot with an empty one).  skip: a bit for every element that is one of the
    // teacher's places.
    __device__ __forceinline__ void add(const float (&x)[VEC], unsigned skip)
    {
        float e[VEC], sum, h;
        for (;;) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) e[i] = at.soft(x[i]);
            sum = e[0];
#pragma unroll
            for (int i = 1; i < VEC; ++i) sum += e[i];
            bool high = !(sum <= 0x1p24f);              // NaN among them
            if constexpr (HARD == HARD_EXP) {
                h = at.hard(x[0]);
#pragma unroll
                for (int i = 1; i < VEC; ++i) h += at.hard(x[i]);
                high = high || !(h <= 0x1p24f);
            }
            if (at.ref > -INFINITY && !__any(high)) break;      // uniform for the wavefront, and nearly always
            if (at.by_difference()) {                   // uniform
#pragma unroll
                for (int i = 0; i < VEC; ++i) e[i] = exp2_fast((x[i] - at.ref) * q.c);
                sum = e[0];
#pragma unroll
                for (int i = 1; i < VEC; ++i) sum += e[i];
                high = !(sum <= 0x1p24f);
                if constexpr (HARD == HARD_EXP) {
                    h = exp2_fast((x[0] - at.ref) * q.c1);
#pragma unroll
                    for (int i = 1; i < VEC; ++i) h += exp2_fast((x[i] - at.ref) * q.c1);
                    high = high || !(h <= 0x1p24f);
                }
                if (!__any(high)) break;
            }
            float t = x[0];
#pragma unroll
            for (int i = 1; i < VEC; ++i) t = fmaxf(t, x[i]);
            t = uniform(wave_max(t));
            if (!(t > at.ref)) break;
            const Reference<VEC> old = at;
            at.set(t, q);
            const float f = change(old, at, q.c, old.lost, at.lost), f1 = change(old, at, q.c1, old.lost1, at.lost1);
            st *= f;
            if constexpr (TAIL) some = some || so > 0.f;
            so *= f;
            s1 *= f1;
        }
        st += sum;
        if constexpr (HARD == HARD_EXP) s1 += h;
        if constexpr (HARD == HARD_SQUARE) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) s1 = fmaf(e[i], e[i], s1);
        }
        if constexpr (TAIL) {
            if (skip) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) so += (skip >> i & 1) ? 0.f : e[i];
            } else so += sum;
        }
    }
    // For whole wavefronts, after some slots: calls look() as long as no exponential outside the teacher's places has been above 0 and no look at
    // the slots has found a logit there that is not masked.  In all but masked rows that ends with the first slots.
    template <typename L> __device__ __forceinline__ void until_settled(L look)
    {
        if (!TAIL || settled) return;
        if (!__any(so > 0.f)) look();
        settled = __any(some || so > 0.f);
    }
    // what sums relative to `old` are multiplied with to be relative to `now`
    __device__ static __forceinline__ float change(const Reference<VEC> &old, const Reference<VEC> &now, float c, float old_lost, float now_lost)
    {
        return old.ref == -INFINITY ? 1.f : exp2_fast((old.ref - now.ref) * c - old_lost + now_lost);
    }
    // the sums of the threads of a block relative to their largest reference, in a fixed order; part: one float4 per wavefront
    template <int BLOCK> __device__ __forceinline__ float4 combine(float4 *part)
    {
        constexpr int WAVES = BLOCK / 64;
        const float f = exp2_fast(-at.lost), f1 = exp2_fast(-at.lost1);
        if constexpr (TAIL) so = some && so == 0.f ? OUTSIDE_TINY : so;
        float4 w = make_float4(at.ref, wave_sum(st) * f, wave_sum(s1) * f1, wave_sum(so) * f);
        static_assert(WAVES > 1, "part is used");
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = w;
        __syncthreads();
        w = part[threadIdx.x & (WAVES - 1)];
        float M = w.x;
#pragma unroll
        for (int o = WAVES / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
        float4 all = make_float4(M, 0.f, 0.f, 0.f);
        join(all, w, q);
#pragma unroll
        for (int o = WAVES / 2; o > 0; o >>= 1) {
            all.y += __shfl_xor(all.y, o);
            all.z += __shfl_xor(all.z, o);
            all.w += __shfl_xor(all.w, o);
        }
        if constexpr (HARD == HARD_PLAIN) all.z = all.y;
        return all;
    }
    // adds the sums of a part, relative to its own reference, to those relative to w.x, which is at least as large
    __device__ static __forceinline__ void join(float4 &w, const float4 &p, const Scales &q)
    {
        const float d = p.x == w.x || p.x == -INFINITY ? 0.f : p.x - w.x;      // a part of masked places has sums of 0
        const float f = exp2_fast(d * q.c);
        w.y += p.y * f;
        w.z += p.z * exp2_fast(d * q.c1);
        if constexpr (TAIL) w.w = fmaxf(w.w + p.w * f, p.w > 0.f ? OUTSIDE_TINY : 0.f);
    }
};

}  // namespace easgd
