// Gradients of rows of logits: where they go, and what is checked about them.
#pragma once
#include "logits.h"

namespace easgd {

// The rows of the gradient, which may start at another alignment than the logits': whole slots where both agree (the
// usual case: SAME), else element by element.
template <int DT> struct GradRow {
    using Type = LogitType<DT>;
    static constexpr int VEC = Type::VEC;
    typename Type::Stored *row;         // element 0
    int shift, V;
    bool same;
    __device__ __forceinline__ GradRow(void *dlogits, size_t dld, int V, size_t r, const Row<DT> &in)
    {
        const Row<DT> out(dlogits, r, dld, V);
        row = out.base + out.shift;
        same = out.shift == in.shift;
        shift = in.shift;
        this->V = V;
    }
    // the gradient of slot s of the logits' grid
    __device__ __forceinline__ void store(int s, const float (&x)[VEC], bool full) const
    {
        const int j = s * VEC - shift;
        if (same && full) {
            typedef unsigned Four __attribute__((ext_vector_type(4)));
            const uint4 p = Type::pack(x);
            const Four v = {p.x, p.y, p.z, p.w};
            __builtin_nontemporal_store(v, reinterpret_cast<Four *>(row + j));
            return;
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if ((unsigned)(j + i) < (unsigned)V) row[j + i] = Type::narrow(x[i]);
    }
    // the gradient of slot `from` + thread, which is full, where the alignments agree: a uniform address and an offset
    __device__ __forceinline__ void store_at(int from, const float (&x)[VEC]) const
    {
        typedef unsigned Four __attribute__((ext_vector_type(4)));
        const uint4 p = Type::pack(x);
        const Four v = {p.x, p.y, p.z, p.w};
        __builtin_nontemporal_store(v, reinterpret_cast<Four *>(row + from * VEC - shift) + (unsigned)threadIdx.x);
    }
    __device__ __forceinline__ void put(int j, float d) const { row[j] = Type::narrow(d); }
    // 0 for slots first + thread, first + thread + block, ... below last
    __device__ __forceinline__ void clear(int last, int block, int first = 0) const
    {
        const float zero[VEC] = {};
        for (int s = first + threadIdx.x; s < last; s += block) store(s, zero, s * VEC >= shift && (s + 1) * VEC <= shift + V);
    }
};

static inline int check_gradient(const char *name, const void *dlogits, int dtype, size_t rows, int V, size_t dld, float scale)
{
    if (!std::isfinite(scale)) return fail(EASGD_EINVAL, "%s: scale must be finite", name);
    if (dld < (size_t)V) return fail(EASGD_EINVAL, "%s: dld (%zu) < V (%d)", name, dld, V);
    if (rows > 1 && dld > ((size_t)1 << 60) / rows) return fail(EASGD_ERANGE, "%s: rows * dld too large", name);
    if (!aligned_to(dlogits, dtype_bytes(dtype))) return fail(EASGD_EINVAL, "%s: dlogits must be aligned to its elements (%zu bytes)", name, dtype_bytes(dtype));
    return EASGD_OK;
}

// Whether a row of logits and one of dlogits share memory: blocks read a row, or parts of others, while they store.  Rows that
// alternate (the two halves of wider rows, say) share none; at two strides the whole ranges have to be apart.
static inline bool rows_overlap(const void *logits, size_t ld, const void *dlogits, size_t dld, int V, size_t rows, size_t size)
{
    const uintptr_t in = reinterpret_cast<uintptr_t>(logits), out = reinterpret_cast<uintptr_t>(dlogits);
    const size_t row = (size_t)V * size;
    if (in + (rows - 1) * ld * size + row <= out || out + (rows - 1) * dld * size + row <= in) return false;
    if (rows == 1 || ld != dld) return true;
    const size_t pitch = ld * size, apart = in < out ? (out - in) % pitch : (in - out) % pitch;
    return apart < row || pitch - apart < row;
}

}  // namespace easgd
