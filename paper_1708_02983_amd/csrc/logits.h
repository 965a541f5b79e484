// Rows of logits in device memory: element types, 128-bit access at any alignment, the order of logits, reductions over
// a block.  Shared by the kernels that work on rows of logits (top logits, distillation, sampling).
#pragma once
#include <cfloat>
#include <cmath>
#include <type_traits>
#include "common.h"

namespace easgd {

static constexpr int LOGITS_MAX_V = 1 << 20;      // an index fits 20 bits of an order word
static constexpr size_t LOGITS_MAX_ROWS = ((size_t)1 << 22) - 1;
static constexpr int LOGITS_MAX_TOP = EASGD_MAX_TOP;

// one of four words by number, without an indexed register
__device__ __forceinline__ unsigned word_of(const uint4 &v, int i)
{
    const unsigned low = i & 1 ? v.y : v.x, high = i & 1 ? v.w : v.z;
    return i & 2 ? high : low;
}

// Element types: 128 bits hold VEC elements; every type widens to fp32 without loss.
template <int DT> struct LogitType;
template <> struct LogitType<EASGD_F32> {
    using Stored = float;
    static constexpr int VEC = 4;
    static constexpr unsigned NEG_INF = 0xff800000u;
    __device__ static __forceinline__ float widen(Stored b) { return b; }
    __device__ static __forceinline__ float pick(const uint4 &v, int j) { return __uint_as_float(word_of(v, j)); }
    __device__ static __forceinline__ void unpack(const uint4 &v, float (&x)[VEC])
    {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[VEC])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static __forceinline__ Stored narrow(float x) { return x; }
    __device__ static __forceinline__ unsigned bits(Stored b) { return __float_as_uint(b); }
};
template <> struct LogitType<EASGD_BF16> {
    using Stored = __bf16;
    static constexpr int VEC = 8;
    static constexpr unsigned NEG_INF = 0xff80u;
    __device__ static __forceinline__ float widen(Stored b) { return (float)b; }
    __device__ static __forceinline__ float pick(const uint4 &v, int j)
    {
        const unsigned w = word_of(v, j >> 1);
        return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ static __forceinline__ void unpack(const uint4 &v, float (&x)[VEC])
    {
        const unsigned u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[VEC])
    {
        typedef __bf16 Pair __attribute__((ext_vector_type(2)));
        unsigned u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Pair p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};        // one conversion instruction, to nearest even
            u[i] = __builtin_bit_cast(unsigned, p);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    __device__ static __forceinline__ Stored narrow(float x) { return (__bf16)x; }
    __device__ static __forceinline__ unsigned bits(Stored b) { return __builtin_bit_cast(unsigned short, b); }
};
template <> struct LogitType<EASGD_F16> {
    using Stored = _Float16;
    static constexpr int VEC = 8;
    static constexpr unsigned NEG_INF = 0xfc00u;
    __device__ static __forceinline__ float widen(Stored b) { return (float)b; }
    __device__ static __forceinline__ float pick(const uint4 &v, int j)
    {
        return (float)__builtin_bit_cast(_Float16, (unsigned short)(word_of(v, j >> 1) >> (j & 1 ? 16 : 0)));
    }
    __device__ static __forceinline__ void unpack(const uint4 &v, float (&x)[VEC])
    {
        typedef _Float16 Pair __attribute__((ext_vector_type(2)));
        const unsigned u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Pair p = __builtin_bit_cast(Pair, u[i]);
            x[2 * i] = (float)p[0];
            x[2 * i + 1] = (float)p[1];
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[VEC])
    {
        typedef _Float16 Pair __attribute__((ext_vector_type(2)));
        unsigned u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Pair p = {(_Float16)x[2 * i], (_Float16)x[2 * i + 1]};
            u[i] = __builtin_bit_cast(unsigned, p);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    __device__ static __forceinline__ Stored narrow(float x) { return (_Float16)x; }
    __device__ static __forceinline__ unsigned bits(Stored b) { return __builtin_bit_cast(unsigned short, b); }
};

// One row as a sequence of slots of 128 bits on the 16-byte grid of memory, in index order: element j sits at place
// j + shift, slot s holds places [s*VEC, (s+1)*VEC).  A row may start at any element's address (an odd stride puts every
// row at another alignment), so the first and the last slot may be partial: they are put together from single elements,
// places outside the row hold -inf, and nothing outside the row is read or written.
template <int DT> struct Row {
    using Type = LogitType<DT>;
    using Stored = typename Type::Stored;
    static constexpr int VEC = Type::VEC;
    Stored *base;         // the 16-byte boundary at or before element 0 (never dereferenced before element 0)
    int shift, end;       // the row's places are [shift, end)
    int slots;

    __device__ __forceinline__ Row(const void *matrix, size_t row, size_t ld, int V)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(matrix) + row * ld * sizeof(Stored);
        shift = (int)((at & 15u) / sizeof(Stored));
        base = reinterpret_cast<Stored *>(at & ~(uintptr_t)15);
        end = shift + V;
        slots = (end + VEC - 1) / VEC;
    }
    __device__ __forceinline__ int first_full() const { return shift ? 1 : 0; }
    __device__ __forceinline__ int end_full() const { return end / VEC; }         // full slots are [first_full, end_full)
    __device__ __forceinline__ bool full(int s) const { return s * VEC >= shift && (s + 1) * VEC <= end; }
    __device__ __forceinline__ uint4 load_full(int s) const { return reinterpret_cast<const uint4 *>(base)[s]; }
    // for what is read once and no more by anyone soon
    __device__ __forceinline__ uint4 load_once(int s) const
    {
        typedef unsigned Four __attribute__((ext_vector_type(4)));
        const Four v = __builtin_nontemporal_load(reinterpret_cast<const Four *>(base) + s);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    __device__ __forceinline__ float load_one(int j) const { return Type::widen(base[shift + j]); }
    __device__ __forceinline__ uint4 load(int s) const
    {
        if (full(s)) return load_full(s);
        unsigned e[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int p = s * VEC + i;
            e[i] = (p >= shift && p < end) ? Type::bits(base[p]) : Type::NEG_INF;
        }
        if constexpr (VEC == 4) return make_uint4(e[0], e[1], e[2], e[3]);
        else return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4 % VEC] | e[5 % VEC] << 16, e[6 % VEC] | e[7 % VEC] << 16);
    }
    // slot s, or an empty one from `last` on: for lanes of a wavefront on consecutive slots, whose place is looked at once
    __device__ __forceinline__ uint4 load_wave(int s, int last) const
    {
        const int first = __builtin_amdgcn_readfirstlane(s - (int)(threadIdx.x & 63));
        if (first * VEC >= shift && first + 64 <= last && (first + 64) * VEC <= end) return load_full(s);
        return s < last ? load(s) : empty();
    }
    __device__ static __forceinline__ uint4 empty()
    {
        constexpr unsigned two = VEC == 4 ? Type::NEG_INF : Type::NEG_INF << 16 | Type::NEG_INF;
        return make_uint4(two, two, two, two);
    }
    // index of the element at place i of slot s
    __device__ __forceinline__ int index(int s, int i) const { return s * VEC + i - shift; }
};

// The order of logits: larger logits first, equal ones by ascending index.  A logit's key is a whole number that orders
// as the logit does (both zeros are one value); -inf and NaN have key 0 and are never taken.  The order word of an
// element, key << 32 | ~index, is unique in a row, so "the first n of the order" is "all words >= the n-th".
__device__ __forceinline__ unsigned logit_key(float x)
{
    const unsigned b = __float_as_uint(x + 0.f);
    const unsigned key = b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
    return x > -INFINITY ? key : 0u;
}
__device__ __forceinline__ float key_logit(unsigned key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ unsigned long long order_word(unsigned key, int index)
{
    return (unsigned long long)key << 32 | (unsigned)~index;
}
static constexpr unsigned long long FIRST_WORD = 1ull << 32;      // below it: key 0

// 2^x of the hardware (about one unit in the last place, results below the smallest normal number are 0)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
static constexpr double LOG2E = 1.44269504088896340736;

// ---- reductions over a block of BLOCK threads, in fixed orders ---------------------------------------------------
template <typename T> __device__ __forceinline__ T wave_sum(T v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
// the one value among the lanes that is not 0 (or 0)
__device__ __forceinline__ float wave_only(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float other = __shfl_xor(v, o);
        v = v != 0.f ? v : other;
    }
    return v;
}
// scratch: one T per wavefront; ends with every thread holding the sum, and with scratch free again
template <int BLOCK, typename T> __device__ __forceinline__ T block_sum(T v, T *scratch)
{
    constexpr int WAVES = BLOCK / 64;
    static_assert((WAVES & (WAVES - 1)) == 0, "the wavefronts' values are joined in a tree");
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = scratch[threadIdx.x & (WAVES - 1)];         // one load and a tree: registers are scarce where rows are held in them
#pragma unroll
        for (int o = WAVES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
        __syncthreads();
    }
    return v;
}
template <int BLOCK> __device__ __forceinline__ float block_max(float v, float *scratch)
{
    constexpr int WAVES = BLOCK / 64;
    v = wave_max(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = scratch[threadIdx.x & (WAVES - 1)];
#pragma unroll
        for (int o = WAVES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
        __syncthreads();
    }
    return v;
}

// calls f with the element type as a constant
template <typename F> static void by_dtype(int dtype, F f)
{
    if (dtype == EASGD_F32) f(std::integral_constant<int, EASGD_F32>{});
    else if (dtype == EASGD_BF16) f(std::integral_constant<int, EASGD_BF16>{});
    else f(std::integral_constant<int, EASGD_F16>{});
}

static inline size_t dtype_bytes(int dtype) { return dtype == EASGD_F32 ? 4 : 2; }

// What every call on rows of logits checks about them; EASGD_OK, or the error with its message set.
static inline int check_logits(const char *name, const void *logits, int dtype, size_t rows, int V, size_t ld)
{
    if (dtype != EASGD_F32 && dtype != EASGD_BF16 && dtype != EASGD_F16) return fail(EASGD_EINVAL, "%s: unknown element type %d", name, dtype);
    if (V < 1) return fail(EASGD_EINVAL, "%s: V (%d) < 1", name, V);
    if (V > LOGITS_MAX_V) return fail(EASGD_ERANGE, "%s: V (%d) above %d", name, V, LOGITS_MAX_V);
    if (ld < (size_t)V) return fail(EASGD_EINVAL, "%s: ld (%zu) < V (%d)", name, ld, V);
    if (rows > LOGITS_MAX_ROWS) return fail(EASGD_ERANGE, "%s: more than %zu rows", name, LOGITS_MAX_ROWS);       // a grid has fewer than 2^32 threads
    if (rows > 1 && ld > ((size_t)1 << 60) / rows) return fail(EASGD_ERANGE, "%s: rows * ld too large", name);
    if (rows > 0 && !logits) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(logits, dtype_bytes(dtype))) return fail(EASGD_EINVAL, "%s: logits must be aligned to their elements (%zu bytes)", name, dtype_bytes(dtype));
    return EASGD_OK;
}
// Slots of a row of V elements at the worst alignment
static inline int most_slots(int dtype, int V)
{
    const int vec = dtype == EASGD_F32 ? 4 : 8;
    return (V + 2 * (vec - 1)) / vec;
}
static inline int check_workspace(const char *name, const void *workspace, size_t bytes, size_t need)
{
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || bytes < need))
        return fail(EASGD_EWORKSPACE, "%s: workspace must be 256-byte aligned and hold %zu bytes (got %zu)", name, need, bytes);
    return EASGD_OK;
}
static inline int check_temperature(const char *name, float T)
{
    if (!(T >= 1e-6f && T <= 1e6f)) return fail(EASGD_EINVAL, "%s: temperature must be in [1e-6, 1e6], got %g", name, (double)T);
    return EASGD_OK;
}

}  // namespace easgd
