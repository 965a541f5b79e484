// Distillation from a teacher's top logits: the loss of every row and its gradient.
//
// Per row (see include/easgd.h for the definition):  with m = max z, e_j = exp((z_j - m)/T), h_j = exp(z_j - m),
//   ST = sum e_j, SO = sum of e_j outside the teacher's places, S1 = sum h_j,
//   KL   = sum_i p_i (log p_i - (z[t_i] - m)/T + log ST)  (+ r (log r - log SO + log ST)),   CE = m - z_y + log S1
//   grad = soft (c e_j / ST - target_j - [j outside] r e_j / SO) + up hard (h_j / S1 - [j = y]),  soft = up (1 - hard) T
// so a row is read for its maximum and its sums, and once more for its gradient.  Bound: HBM (each logit once in, each
// gradient once out), with the vector ALUs close behind (an exponential takes four issue slots, and either pass has one).
#include "logits.h"

namespace easgd {

struct DistillArgs {
    const void *logits;
    size_t ld;
    int V, k;
    const int *indices;
    const float *values, *teacher_lse;
    const int *labels;
    float temperature, hard;
    float *loss, *state;
    const float *dloss;
    float scale;
    void *dlogits;
    size_t dld;
    float4 *partial;          // [rows][segments]: (m, ST, S1, SO) of a part of a row
    int segments, seg_slots;  // slots of a part of a row
};

enum { DISTILL_LOSS = 1, DISTILL_GRAD = 2, DISTILL_BOTH = 3 };

// ---- exponentials of a row at both temperatures ------------------------------------------------------------------
// h_j is a power of e_j where T is 1, 2 or 4: one or two multiplications in the place of an exponential.
enum { HARD_NONE = 0, HARD_SAME = 1, HARD_SQUARE = 2, HARD_FOURTH = 3, HARD_EXP = 4 };

struct Scales {
    float c, c1;              // log2(e) / T, log2(e)
    float margin;             // logits this far above the reference make exponentials of 2^24 at most
    int hard;                 // where h_j comes from; HARD_NONE: nobody asks for it
    __device__ __forceinline__ Scales(const DistillArgs &a)
    {
        c = (float)(LOG2E / (double)a.temperature);
        c1 = (float)LOG2E;
        margin = 24.f / fmaxf(c, c1);
        hard = !(a.hard > 0.f) ? HARD_NONE : a.temperature == 1.f ? HARD_SAME : a.temperature == 2.f ? HARD_SQUARE :
               a.temperature == 4.f ? HARD_FOURTH : HARD_EXP;
    }
    __device__ __forceinline__ float soft(float d) const { return exp2_fast(d * c); }
};

// Running sums of a thread, relative to a reference near the maximum that its wavefront shares: it is moved only when
// a logit exceeds it by 24 binary orders of magnitude (sums of 2^20 such terms are far from fp32's end), so that the
// loop over a row has one comparison for it instead of a rescaling per 128 bits.
template <int VEC, bool TAIL> struct RowSums {
    float ref = -INFINITY, top = -INFINITY, st = 0.f, s1 = 0.f, so = 0.f;

    // Whole wavefronts call it (lanes without a slot with an empty one).  skip: a bit for every element that is one of the
    // teacher's places.
    __device__ __forceinline__ void add(const float (&x)[VEC], unsigned skip, const Scales &q)
    {
        float t = x[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) t = fmaxf(t, x[i]);
        top = fmaxf(top, t);
        if (__any(t > ref + q.margin)) {                // uniform for the wavefront
            const float up = fmaxf(ref, wave_max(t));
            const float f = ref == -INFINITY ? 0.f : q.soft(ref - up);
            st *= f;
            so *= f;
            s1 *= ref == -INFINITY ? 0.f : exp2_fast((ref - up) * q.c1);
            ref = up;
        }
        const float m = ref == -INFINITY ? 0.f : ref;   // nothing but -inf so far: every exponential is 0
        float e[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) e[i] = q.soft(x[i] - m);
        float sum = e[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) sum += e[i];
        st += sum;
        if constexpr (TAIL) {
            if (skip) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) so += (skip >> i & 1) ? 0.f : e[i];
            } else so += sum;
        }
        if (q.hard >= HARD_SQUARE) {                    // uniform
            if (q.hard == HARD_EXP) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) s1 += exp2_fast((x[i] - m) * q.c1);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float e2 = e[i] * e[i];
                    s1 = q.hard == HARD_SQUARE ? s1 + e2 : fmaf(e2, e2, s1);
                }
            }
        }
    }
    // the sums of the threads of a block relative to the maximum, in a fixed order; part: one float4 per wavefront
    template <int BLOCK> __device__ __forceinline__ float4 combine(const Scales &q, float4 *part)
    {
        constexpr int WAVES = BLOCK / 64;
        const float m = wave_max(top);
        const float f = m == -INFINITY ? 1.f : ref == -INFINITY ? 0.f : q.soft(ref - m);
        const float f1 = m == -INFINITY ? 1.f : ref == -INFINITY ? 0.f : exp2_fast((ref - m) * q.c1);
        float4 w = make_float4(m, wave_sum(st) * f, wave_sum(s1) * f1, wave_sum(so) * f);
        if constexpr (WAVES == 1) return w;
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
        return all;
    }
    // adds the sums of a part, relative to its own maximum, to those relative to w.x, which is at least as large
    __device__ static __forceinline__ void join(float4 &w, const float4 &p, const Scales &q)
    {
        const float d = p.x == w.x || w.x == -INFINITY ? 0.f : p.x - w.x;
        const float f = q.soft(d);
        w.y += p.y * f;
        w.z += p.z * exp2_fast(d * q.c1);
        w.w += p.w * f;
    }
};

// ---- the teacher ---------------------------------------------------------------------------------------------------
// What a row's teacher asks for.  Its 64-bit numbers live in LDS: the registers hold the row.
struct TeacherLds {
    int index[LOGITS_MAX_TOP];             // -1: slot not used
    double log_p[LOGITS_MAX_TOP], p[LOGITS_MAX_TOP];
    double mass, rest;                     // sum of p; what it leaves over (0 without a teacher's log-sum-exp)
    double part[16];
    float fpart[16];
};

// Slot i goes through thread i; returns its place.
template <int BLOCK, bool TAIL>
__device__ __forceinline__ int read_teacher(const DistillArgs &a, size_t r, TeacherLds &lds)
{
    static_assert(BLOCK >= LOGITS_MAX_TOP, "one thread per slot of the teacher");
    const int tid = threadIdx.x;
    const double T = (double)a.temperature;
    int place = -1;
    double logit = -INFINITY;
    if (tid < a.k) {
        place = a.indices[r * a.k + tid];
        const float v = a.values[r * a.k + tid];
        if ((unsigned)place >= (unsigned)a.V) place = -1;
        else logit = (double)v / T;
        lds.index[tid] = place;
    }
    double lse;
    if constexpr (TAIL) lse = (double)a.teacher_lse[r];
    else {
        const float top = block_max<BLOCK>((float)logit, lds.fpart);
        const double total = block_sum<BLOCK>(place >= 0 && top > -INFINITY ? exp(logit - (double)top) : 0.0, lds.part);
        lse = (double)top + log(total);
        if (!(top > -INFINITY)) lse = isnan(total) ? (double)NAN : 0.0;      // no used slot, or all masked: no probability anywhere
    }
    const double log_p = logit - lse, p = place >= 0 ? exp(log_p) : 0.0;
    if (tid < a.k) {
        lds.log_p[tid] = log_p;
        lds.p[tid] = p;
    }
    const double mass = block_sum<BLOCK>(p, lds.part);
    if (tid == 0) {
        lds.mass = mass;
        lds.rest = TAIL && mass < 1.0 ? 1.0 - mass : 0.0;
    }
    __syncthreads();
    return place;
}

// A bit per element of the places [first, first + 32 * words) on the row's 16-byte grid: the teacher's places.
__device__ __forceinline__ void mark_places(unsigned *bits, int words, int first, int place, int shift, int block)
{
    for (int w = threadIdx.x; w < words; w += block) bits[w] = 0;
    __syncthreads();
    const int at = place + shift - first;
    if (place >= 0 && at >= 0 && at < 32 * words) atomicOr(&bits[at >> 5], 1u << (at & 31));
    __syncthreads();
}
template <int VEC> __device__ __forceinline__ unsigned marks_of(const unsigned *bits, int slot)
{
    return (bits[slot * VEC >> 5] >> (slot * VEC & 31)) & ((1u << VEC) - 1);
}

// The row's loss from its sums (M, ST, S1, SO); every thread of the block calls it.
template <int BLOCK>
__device__ __forceinline__ void write_loss(const DistillArgs &a, size_t r, int place, float z_place, float z_label, bool padding,
                                           const float4 &s, TeacherLds &lds)
{
    const double T = (double)a.temperature;
    const bool none = padding || s.y == 0.f;           // padding, or every logit masked
    const double log_st = log((double)s.y);
    const double p = place >= 0 ? lds.p[threadIdx.x] : 0.0;
    double term = 0.0;
    if (!none && p > 0.0) term = p * (lds.log_p[threadIdx.x] - (((double)z_place - (double)s.x) / T - log_st));
    if (isnan(p)) term = p;
    double kl = block_sum<BLOCK>(term, lds.part);
    if (threadIdx.x != 0) return;
    if (lds.rest > 0.0 && s.w > 0.f) kl += lds.rest * (log(lds.rest) - log((double)s.w) + log_st);
    double loss = 0.0;
    if (!none) {
        if (a.hard < 1.f) loss = (1.0 - (double)a.hard) * T * T * kl;
        if (a.hard > 0.f) loss += (double)a.hard * (((double)s.x - (double)z_label) + log((double)s.z));
        if (isnan(s.y)) loss = NAN;
    }
    a.loss[r] = (float)loss;
    if (a.state) reinterpret_cast<float4 *>(a.state)[r] = padding ? make_float4(0.f, 0.f, 0.f, 0.f) : s;
}

// ---- the gradient ----------------------------------------------------------------------------------------------------
// The factors of a row's gradient: outside the places that the teacher or the label names it is fq e_j + f1 h_j.
struct Factors {
    double soft, up_hard, cover, outside;
    __device__ __forceinline__ Factors(const DistillArgs &a, size_t r, const TeacherLds &teacher, const float4 &s)
    {
        const double up = (double)a.scale * (a.dloss ? (double)a.dloss[r] : 1.0);
        const double rest = s.w > 0.f ? teacher.rest : 0.0;
        soft = up * (1.0 - (double)a.hard) * (double)a.temperature;
        up_hard = up * (double)a.hard;
        cover = teacher.mass + rest;
        outside = rest > 0.0 ? cover - rest * (double)s.y / (double)s.w : cover;
    }
};
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
struct Slope {
    float fq, f1, m;
    bool none;                 // nothing to learn: the gradient is 0
    __device__ __forceinline__ Slope(const DistillArgs &a, size_t r, const TeacherLds &teacher, bool padding, const float4 &s)
    {
        none = padding || uniform(s.y) == 0.f;
        const Factors f(a, r, teacher, s);
        fq = uniform((float)(f.soft * f.outside / (double)s.y));
        f1 = a.hard > 0.f ? uniform((float)(f.up_hard / (double)s.z)) : 0.f;
        m = uniform(s.x);
    }
};

template <int VEC> __device__ __forceinline__ void slope_of(float (&x)[VEC], const Slope &g, const Scales &q)
{
    if (g.none) {                                      // uniform
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = 0.f;
        return;
    }
    if (q.hard == HARD_EXP) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float d = x[i] - g.m;
            x[i] = fmaf(g.f1, exp2_fast(d * q.c1), g.fq * q.soft(d));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float e = q.soft(x[i] - g.m);
        if (q.hard == HARD_NONE) x[i] = g.fq * e;
        else if (q.hard == HARD_SAME) x[i] = (g.fq + g.f1) * e;
        else if (q.hard == HARD_SQUARE) x[i] = e * fmaf(g.f1, e, g.fq);
        else x[i] = e * fmaf(g.f1, e * (e * e), g.fq);
    }
}

// The rows of the gradient, which may start at another alignment than the logits': whole slots where both agree (the
// usual case: SAME), else element by element.
template <int DT> struct GradRow {
    using Type = LogitType<DT>;
    static constexpr int VEC = Type::VEC;
    typename Type::Stored *row;         // element 0
    int shift, V;
    bool same;
    __device__ __forceinline__ GradRow(const DistillArgs &a, size_t r, const Row<DT> &in)
    {
        const Row<DT> out(a.dlogits, r, a.dld, a.V);
        row = out.base + out.shift;
        same = out.shift == in.shift;
        shift = in.shift;
        V = a.V;
    }
    // the gradient of slot s of the logits' grid
    __device__ __forceinline__ void store(int s, const float (&x)[VEC], bool full) const
    {
        const int j = s * VEC - shift;
        if (same && full) {
            *reinterpret_cast<uint4 *>(row + j) = Type::pack(x);
            return;
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if ((unsigned)(j + i) < (unsigned)V) row[j + i] = Type::narrow(x[i]);
    }
    __device__ __forceinline__ void put(int j, float d) const { row[j] = Type::narrow(d); }
};

// The places that the teacher or the label names, within elements [j0, j1) (j0 may lie before the row): each once, by the
// first slot that names it, after a barrier behind the stores of all others.
template <int DT>
__device__ __forceinline__ void name_places(const DistillArgs &a, size_t r, const Row<DT> &row, const GradRow<DT> &out, int place, int label,
                                            const float4 &s, const TeacherLds &lds, int j0, int j1)
{
    const bool labelled = a.hard > 0.f;
    int at = -1;
    double target = 0.0;
    if (place >= max(j0, 0) && place < j1) {
        at = place;
        for (int i = 0; i < a.k; ++i) {
            if (lds.index[i] != place) continue;
            if (i < (int)threadIdx.x) at = -1;
            target += lds.p[i];
        }
    }
    const Factors f(a, r, lds, s);
    auto name = [&](int j, bool top, double goal) {
        const double x = (double)row.load_one(j) - (double)s.x;
        double d = f.soft * ((top ? f.cover : f.outside) * exp(x / (double)a.temperature) / (double)s.y - goal);
        if (f.up_hard != 0.0) d += f.up_hard * (exp(x) / (double)s.z - (labelled && j == label ? 1.0 : 0.0));
        out.put(j, (float)d);
    };
    bool alone = labelled && threadIdx.x == blockDim.x - 1 && label >= j0 && label < j1;    // a label that no slot names
    if (alone)
        for (int i = 0; i < a.k; ++i) alone = alone && lds.index[i] != label;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        const int j = turn == 0 ? at : alone ? label : -1;
        if (j >= 0) name(j, turn == 0, target);
        target = 0.0;
    }
}

// ---- loss, and gradient with GRAD, of whole rows, a block each -----------------------------------------------------
// The first NV * BLOCK slots of a row are requested at once and stay in registers between the two passes over it, so
// that up to 256 KB of a row are read once; what is longer is read again.
template <int DT, int BLOCK, int NV, bool TAIL, bool GRAD>
__global__ __launch_bounds__(BLOCK) void distill_rows_kernel(DistillArgs a)
{
    constexpr int VEC = Row<DT>::VEC;
    using Type = LogitType<DT>;
    extern __shared__ unsigned in_top[];
    __shared__ TeacherLds lds;
    __shared__ float4 part[BLOCK / 64];
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const Scales q(a);
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;

    // full slots [f0, f1): thread t has f0 + t + i * BLOCK; threads 0 and 1 have the partial slots at the row's ends.  Loops run
    // for whole wavefronts (first is the wavefront's first slot); lanes behind the end hold empty slots.
    const int f0 = row.first_full(), f1 = row.end_full();
    const int first = f0 + __builtin_amdgcn_readfirstlane(tid & ~63);
    uint4 v[NV];
    uint4 edge = make_uint4(0, 0, 0, 0);
    int edge_slot = -1;
    if (tid == 0 && row.shift) edge_slot = 0;
    if (tid == 1 && row.slots > f1 && (row.slots > 1 || !row.shift)) edge_slot = row.slots - 1;
    if (!padding) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int s = f0 + tid + i * BLOCK;
            if (first + i * BLOCK < f1) v[i] = s < f1 ? row.load_full(s) : Row<DT>::empty();
        }
        if (edge_slot >= 0) edge = row.load(edge_slot);
    }
    const int place = read_teacher<BLOCK, TAIL>(a, r, lds);
    float4 sums = make_float4(0.f, 0.f, 0.f, 0.f);
    float z_place = 0.f, z_label = 0.f;
    if (!padding) {                                     // uniform
        if (place >= 0) z_place = row.load_one(place);
        if (tid == 0) z_label = row.load_one(label);
        if constexpr (TAIL) mark_places(in_top, (row.slots * VEC + 31) / 32, 0, place, row.shift, BLOCK);
        RowSums<VEC, TAIL> acc;
        auto add = [&](const uint4 &raw, int s) {
            float x[VEC];
            Type::unpack(raw, x);
            acc.add(x, TAIL ? marks_of<VEC>(in_top, s) : 0u, q);
        };
        if (tid < 64 && __any(edge_slot >= 0)) {        // the first wavefront; lanes without an edge add -inf
            if (edge_slot < 0) edge = Row<DT>::empty();
            add(edge, edge_slot < 0 ? 0 : edge_slot);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (first + i * BLOCK < f1) add(v[i], min(f0 + tid + i * BLOCK, f1 - 1));
        }
        for (int i = NV; first + i * BLOCK < f1; ++i) {
            const int s = f0 + tid + i * BLOCK;
            add(s < f1 ? row.load_full(s) : Row<DT>::empty(), min(s, f1 - 1));
        }
        sums = acc.template combine<BLOCK>(q, part);
        if (q.hard == HARD_SAME) sums.z = sums.y;
    }
    if constexpr (!GRAD) {
        write_loss<BLOCK>(a, r, place, z_place, z_label, padding, sums, lds);
        return;
    }
    const GradRow<DT> out(a, r, row);
    const Slope g(a, r, lds, padding, sums);
    auto put = [&](const uint4 &raw, int s, bool full) {
        float x[VEC];
        Type::unpack(raw, x);
        slope_of<VEC>(x, g, q);
        out.store(s, x, full);
    };
    if (edge_slot >= 0) put(edge, edge_slot, false);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int s = f0 + tid + i * BLOCK;
        if (s < f1) put(v[i], s, true);
    }
    for (int s = f0 + tid + NV * BLOCK; s < f1; s += BLOCK) put(g.none ? make_uint4(0, 0, 0, 0) : row.load_full(s), s, true);
    write_loss<BLOCK>(a, r, place, z_place, z_label, padding, sums, lds);       // its barriers stand between the stores above and below
    if (!g.none) name_places<DT>(a, r, row, out, place, label, sums, lds, 0, a.V);
}

// ---- few rows: sums of parts of rows ----------------------------------------------------------------------------------
template <int DT, int BLOCK, bool TAIL>
__global__ __launch_bounds__(BLOCK) void distill_sums_kernel(DistillArgs a)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    using Type = LogitType<DT>;
    extern __shared__ unsigned in_top[];
    __shared__ float4 part[BLOCK / 64];
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const Scales q(a);
    if (a.labels && (unsigned)a.labels[r] >= (unsigned)a.V) return;
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    if constexpr (TAIL) {
        int place = -1;
        if (tid < a.k) place = a.indices[r * a.k + tid];
        if ((unsigned)place >= (unsigned)a.V) place = -1;
        mark_places(in_top, (a.seg_slots * VEC + 31) / 32, s0 * VEC, place, row.shift, BLOCK);
    }
    RowSums<VEC, TAIL> acc;
    auto add = [&](const uint4 &raw, int s) {
        float x[VEC];
        Type::unpack(raw, x);
        acc.add(x, TAIL ? marks_of<VEC>(in_top, s - s0) : 0u, q);
    };
    const int lead = __builtin_amdgcn_readfirstlane(tid & ~63);
    int s = s0 + tid;
    for (; s - tid + DEEP * BLOCK <= s1; s += DEEP * BLOCK) {      // uniform
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) v[i] = row.load(s + i * BLOCK);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) add(v[i], s + i * BLOCK);
    }
    for (; s - tid + lead < s1; s += BLOCK) add(s < s1 ? row.load(s) : Row<DT>::empty(), min(s, s1 - 1));      // whole wavefronts
    float4 sums = acc.template combine<BLOCK>(q, part);
    if (q.hard == HARD_SAME) sums.z = sums.y;
    if (tid == 0) a.partial[r * a.segments + seg] = sums;
}

// ---- the losses of rows whose parts were summed apart ----------------------------------------------------------------
template <int DT, bool TAIL>
__global__ __launch_bounds__(256) void distill_join_kernel(DistillArgs a)
{
    __shared__ TeacherLds lds;
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const Scales q(a);
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;
    const int place = read_teacher<256, TAIL>(a, r, lds);
    float4 sums = make_float4(0.f, 0.f, 0.f, 0.f);
    float z_place = 0.f, z_label = 0.f;
    if (!padding) {
        if (place >= 0) z_place = row.load_one(place);
        if (threadIdx.x == 0) z_label = row.load_one(label);
        sums.x = -INFINITY;
        for (int i = 0; i < a.segments; ++i) sums.x = fmaxf(sums.x, a.partial[r * a.segments + i].x);
        for (int i = 0; i < a.segments; ++i) RowSums<4, TAIL>::join(sums, a.partial[r * a.segments + i], q);
    }
    write_loss<256>(a, r, place, z_place, z_label, padding, sums, lds);
}

// ---- backward: gradients of parts of rows ----------------------------------------------------------------------------
template <int DT, int BLOCK, bool TAIL>
__global__ __launch_bounds__(BLOCK) void distill_grad_kernel(DistillArgs a)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    using Type = LogitType<DT>;
    __shared__ TeacherLds lds;
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const Scales q(a);
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    const int place = read_teacher<BLOCK, TAIL>(a, r, lds);
    const float4 sums = reinterpret_cast<const float4 *>(a.state)[r];
    const Slope g(a, r, lds, padding, sums);
    const GradRow<DT> out(a, r, row);
    auto put = [&](const uint4 &raw, int s) {
        float x[VEC];
        Type::unpack(raw, x);
        slope_of<VEC>(x, g, q);
        out.store(s, x, row.full(s));
    };
    int s = s0 + tid;
    if (g.none) {
        for (; s < s1; s += BLOCK) put(make_uint4(0, 0, 0, 0), s);
        return;
    }
    for (; s - tid + DEEP * BLOCK <= s1; s += DEEP * BLOCK) {
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) v[i] = row.load(s + i * BLOCK);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) put(v[i], s + i * BLOCK);
    }
    for (; s < s1; s += BLOCK) put(row.load(s), s);
    __syncthreads();
    name_places<DT>(a, r, row, out, place, label, sums, lds, s0 * VEC - row.shift, s1 * VEC - row.shift);
}

// ---- host --------------------------------------------------------------------------------------------------------------
struct DistillCall {
    const char *name;
    int dtype;
    size_t rows;
    DistillArgs a;
    void *workspace;
    size_t workspace_bytes;
};

static int check_distill(const DistillCall &q, int mode)
{
    const DistillArgs &a = q.a;
    if (int rc = check_logits(q.name, a.logits, q.dtype, q.rows, a.V, a.ld)) return rc;
    if (a.k < 1 || a.k > LOGITS_MAX_TOP) return fail(EASGD_EINVAL, "%s: k must be in [1, %d], got %d", q.name, LOGITS_MAX_TOP, a.k);
    if (int rc = check_temperature(q.name, a.temperature)) return rc;
    if (!(a.hard >= 0.f && a.hard <= 1.f)) return fail(EASGD_EINVAL, "%s: hard must be in [0, 1], got %g", q.name, (double)a.hard);
    if (!a.labels && a.hard != 0.f) return fail(EASGD_EINVAL, "%s: hard = %g needs labels", q.name, (double)a.hard);
    if (q.rows > 0 && (!a.indices || !a.values || ((mode & DISTILL_LOSS) && !a.loss) || (mode == DISTILL_GRAD && !a.state) || ((mode & DISTILL_GRAD) && !a.dlogits)))
        return fail(EASGD_EINVAL, "%s: NULL pointer", q.name);
    if (!aligned_to(a.indices, 4) || !aligned_to(a.values, 4) || !aligned_to(a.teacher_lse, 4) || !aligned_to(a.labels, 4) || !aligned_to(a.loss, 4) ||
        !aligned_to(a.dloss, 4))
        return fail(EASGD_EINVAL, "%s: indices, values, teacher_lse, labels, loss, dloss must be 4-byte aligned", q.name);
    if (!aligned16(a.state)) return fail(EASGD_EINVAL, "%s: state must be 16-byte aligned", q.name);
    if (mode & DISTILL_GRAD) {
        if (!std::isfinite(a.scale)) return fail(EASGD_EINVAL, "%s: scale must be finite", q.name);
        if (a.dld < (size_t)a.V) return fail(EASGD_EINVAL, "%s: dld (%zu) < V (%d)", q.name, a.dld, a.V);
        if (q.rows > 1 && a.dld > ((size_t)1 << 60) / q.rows) return fail(EASGD_ERANGE, "%s: rows * dld too large", q.name);
        if (!aligned_to(a.dlogits, dtype_bytes(q.dtype))) return fail(EASGD_EINVAL, "%s: dlogits must be aligned to its elements (%zu bytes)", q.name, dtype_bytes(q.dtype));
    }
    return EASGD_OK;
}

// Slots of a row of V elements at the worst alignment
static int most_slots(int dtype, int V)
{
    const int vec = dtype == EASGD_F32 ? 4 : 8;
    return (V + 2 * (vec - 1)) / vec;
}

// Into how many parts rows are cut: enough blocks to fill the chip, and at least 1024 slots (four per thread) a part.
static constexpr int SPLIT_BLOCKS = 1024, SPLIT_SLOTS = 1024;
static int segments_of(size_t rows, int slots)
{
    if (rows >= SPLIT_BLOCKS || slots < 2 * SPLIT_SLOTS) return 1;
    const int want = (int)((SPLIT_BLOCKS + rows - 1) / rows), most = slots / SPLIT_SLOTS;
    return want < most ? want : most;
}
static void set_segments(DistillArgs &a, int segments, int slots)
{
    a.segments = segments;
    a.seg_slots = ((slots + segments - 1) / segments + 7) / 8 * 8;      // a multiple of 8: parts of the bit map begin at whole words
}

template <int DT> static void launch_sums(DistillArgs a, size_t rows, hipStream_t s)
{
    constexpr int VEC = LogitType<DT>::VEC;
    const size_t bits = ((size_t)a.seg_slots * VEC + 31) / 32 * 4;
    const dim3 grid((unsigned)(rows * a.segments));
    if (a.teacher_lse) EASGD_LAUNCH((distill_sums_kernel<DT, 256, true>), grid, dim3(256), bits, s, a);
    else EASGD_LAUNCH((distill_sums_kernel<DT, 256, false>), grid, dim3(256), 0, s, a);
    if (a.teacher_lse) EASGD_LAUNCH((distill_join_kernel<DT, true>), dim3((unsigned)rows), dim3(256), 0, s, a);
    else EASGD_LAUNCH((distill_join_kernel<DT, false>), dim3((unsigned)rows), dim3(256), 0, s, a);
}

template <int DT> static void launch_grad(DistillArgs a, size_t rows, hipStream_t s)
{
    const dim3 grid((unsigned)(rows * a.segments));
    if (a.teacher_lse) EASGD_LAUNCH((distill_grad_kernel<DT, 256, true>), grid, dim3(256), 0, s, a);
    else EASGD_LAUNCH((distill_grad_kernel<DT, 256, false>), grid, dim3(256), 0, s, a);
}

template <int DT, int BLOCK, int NV, bool GRAD> static void launch_block(const DistillArgs &a, size_t rows, hipStream_t s)
{
    constexpr int VEC = LogitType<DT>::VEC;
    const size_t bits = ((size_t)a.V + VEC - 1 + 31) / 32 * 4 + 4;
    if (a.teacher_lse) EASGD_LAUNCH((distill_rows_kernel<DT, BLOCK, NV, true, GRAD>), dim3((unsigned)rows), dim3(BLOCK), bits, s, a);
    else EASGD_LAUNCH((distill_rows_kernel<DT, BLOCK, NV, false, GRAD>), dim3((unsigned)rows), dim3(BLOCK), 0, s, a);
}

// The block's size goes by the row's length alone, so that the forward pass adds in the same order with and without the gradient.
template <int DT, bool GRAD> static void launch_rows(const DistillArgs &a, size_t rows, int slots, hipStream_t s)
{
    if (slots <= 256 * 4) launch_block<DT, 256, 4, GRAD>(a, rows, s);
    else if (slots <= 256 * 16) launch_block<DT, 256, 16, GRAD>(a, rows, s);
    else if (slots <= 512 * 16) launch_block<DT, 512, 16, GRAD>(a, rows, s);
    else launch_block<DT, 1024, 16, GRAD>(a, rows, s);
}

// Rows cut into parts: a workspace for the parts' sums, then for the states of the rows.
static size_t split_bytes(size_t rows, int segments) { return segments == 1 ? 0 : (rows * (segments + 1) * sizeof(float4) + 255) / 256 * 256; }

template <int MODE> static int launch_distill(const DistillCall &q, void *stream)
{
    if (int rc = check_distill(q, MODE)) return rc;
    DistillArgs a = q.a;
    const int slots = most_slots(q.dtype, a.V), segments = q.rows ? segments_of(q.rows, slots) : 1;
    set_segments(a, segments, slots);
    if (MODE & DISTILL_LOSS) {
        const size_t need = split_bytes(q.rows, segments);
        if (need && (!q.workspace || (reinterpret_cast<uintptr_t>(q.workspace) & 255u) || q.workspace_bytes < need))
            return fail(EASGD_EWORKSPACE, "%s: workspace must be 256-byte aligned and hold %zu bytes (got %zu)", q.name, need, q.workspace_bytes);
    }
    clear_error();
    if (q.rows == 0) return EASGD_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    a.partial = static_cast<float4 *>(q.workspace);
    by_dtype(q.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if constexpr (MODE == DISTILL_GRAD) launch_grad<DT>(a, q.rows, s);
        else if (segments == 1) launch_rows<DT, MODE == DISTILL_BOTH>(a, q.rows, slots, s);
        else {
            if constexpr (MODE == DISTILL_BOTH) a.state = reinterpret_cast<float *>(a.partial + q.rows * segments);
            launch_sums<DT>(a, q.rows, s);
            if constexpr (MODE == DISTILL_BOTH) launch_grad<DT>(a, q.rows, s);
        }
    });
    return check_launch(q.name);
}

}  // namespace easgd

extern "C" {

size_t easgd_distill_workspace_bytes(size_t rows, int V, int)
{
    using namespace easgd;
    if (rows == 0 || rows > 0x3fffffffull || V < 1 || V > LOGITS_MAX_V) return 0;
    const int most = segments_of(rows, most_slots(EASGD_F32, V)), least = segments_of(rows, most_slots(EASGD_BF16, V));
    return split_bytes(rows, most > least ? most : least);
}

int easgd_distill_loss(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                       const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, float *loss, float *state,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    easgd::DistillCall q = {"easgd_distill_loss", dtype, rows, {}, workspace, workspace_bytes};
    q.a = {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, loss, state, nullptr, 1.f, nullptr, 0, nullptr, 1, 0};
    return easgd::launch_distill<easgd::DISTILL_LOSS>(q, stream);
}

int easgd_distill_grad(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                       const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, const float *state,
                       const float *dloss, float scale, void *dlogits, size_t dld, void *stream)
{
    easgd::DistillCall q = {"easgd_distill_grad", dtype, rows, {}, nullptr, 0};
    q.a = {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, nullptr, const_cast<float *>(state), dloss, scale, dlogits, dld, nullptr, 1, 0};
    return easgd::launch_distill<easgd::DISTILL_GRAD>(q, stream);
}

int easgd_distill(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                  const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, float scale, float *loss,
                  void *dlogits, size_t dld, void *workspace, size_t workspace_bytes, void *stream)
{
    easgd::DistillCall q = {"easgd_distill", dtype, rows, {}, workspace, workspace_bytes};
    q.a = {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, loss, nullptr, nullptr, scale, dlogits, dld, nullptr, 1, 0};
    return easgd::launch_distill<easgd::DISTILL_BOTH>(q, stream);
}

}  // extern "C"
