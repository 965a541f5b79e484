// Distillation from a teacher's top logits: the loss of every row and its gradient.
//
// Per row (see include/easgd.h for the definition):  with m = max z, e_j = exp((z_j - m)/T), h_j = exp(z_j - m),
//   ST = sum e_j, SO = sum of e_j outside the teacher's places, S1 = sum h_j,
//   KL   = sum_i p_i (log p_i - (z[t_i] - m)/T + log ST)  (+ r (log r - log SO + log ST)),   CE = m - z_y + log S1
//   grad = soft (c e_j / ST - target_j - [j outside] r e_j / SO) + up hard (h_j / S1 - [j = y]),  soft = up (1 - hard) T
// so a row is read for its maximum and its sums, and once more for its gradient.  Bound: HBM (each logit once in, each
// gradient once out), with the vector ALUs close behind (an exponential takes four issue slots, and either pass has one).
#include "distill.h"
#include "row_sums.h"

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
    size_t rows;
    int parts;                // logits are the sum of this many matrices (fp32, short rows)
    size_t part_stride;
    float4 *partial;          // [rows][segments]: (m, ST, S1, SO) of a part of a row
    int segments, seg_slots;  // slots of a part of a row
};

enum { DISTILL_LOSS = 1, DISTILL_GRAD = 2, DISTILL_BOTH = 3 };

// ---- the teacher ---------------------------------------------------------------------------------------------------
// What a row's teacher asks for.  Its 64-bit numbers live in LDS: the registers hold the row.
struct TeacherLds {
    __attribute__((aligned(16))) int index[LOGITS_MAX_TOP];       // -1: slot not used
    double log_p[LOGITS_MAX_TOP], p[LOGITS_MAX_TOP];
    double mass, rest;                     // sum of p; what it leaves over (0 without a teacher's log-sum-exp)
    double part[16];
    float fpart[16];
};

// Slot i goes through thread i.
struct Slot {
    int place = -1;            // -1: not used
    float value = 0.f;
    __device__ __forceinline__ void load(const DistillArgs &a, size_t r)
    {
        place = -1;
        if ((int)threadIdx.x < a.k) {
            place = a.indices[r * a.k + threadIdx.x];
            value = a.values[r * a.k + threadIdx.x];
        }
    }
};

// The row's slots and their probabilities into LDS; returns the place of the thread's slot.
template <int BLOCK, bool TAIL>
__device__ __forceinline__ int read_teacher(const DistillArgs &a, size_t r, const Slot &slot, TeacherLds &lds)
{
    static_assert(BLOCK >= LOGITS_MAX_TOP, "one thread per slot of the teacher");
    const int tid = threadIdx.x;
    const double T = (double)a.temperature;
    const int place = (unsigned)slot.place < (unsigned)a.V ? slot.place : -1;
    if (tid < LOGITS_MAX_TOP) lds.index[tid] = place;
    // A masked value has probability 0 whatever the others are; so have all of a row that the teacher masks.  Logits are taken relative to the
    // largest before they are divided and before the logarithm of their sum comes to them: near fp32's ends it would be lost.
    double log_p = -(double)INFINITY;
    if constexpr (TAIL) {
        const float lse = a.teacher_lse[r];
        if (place >= 0 && slot.value != -INFINITY && lse != -INFINITY) log_p = (double)slot.value / T - (double)lse;
    } else {
        const bool live = place >= 0 && slot.value != -INFINITY;
        const float top = block_max<BLOCK>(live ? slot.value : -INFINITY, lds.fpart);
        if (live) log_p = ((double)slot.value - (double)top) / T;
        const double total = block_sum<BLOCK>(live ? exp(log_p) : 0.0, lds.part);
        if (live) log_p -= log(total);
    }
    const double p = place >= 0 ? exp(log_p) : 0.0;
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

// how many of the first k slots name the place (index: 16-byte aligned, -1 behind the last slot up to a multiple of four)
__device__ __forceinline__ int slots_of(const int *index, int k, int place)
{
    int n = 0;
#pragma unroll 4
    for (int i = 0; i < k; i += 4) {
        const int4 q = *reinterpret_cast<const int4 *>(index + i);
        n += (q.x == place) + (q.y == place) + (q.z == place) + (q.w == place);
    }
    return n;
}

// The probabilities of the slots that name a place, added in their order; `first` becomes the first of them.  Every slot is read, named
// or not, so that the reads run ahead (one trip to LDS after the other takes 50 us for 200 slots).
__device__ __forceinline__ double mass_of(const int *index, const double *p, int k, int place, int &first)
{
    double sum = 0.0;
    first = k;
#pragma unroll 8
    for (int i = 0; i < k; ++i) {
        const bool named = index[i] == place;
        const double here = p[i];
        sum += named ? here : 0.0;
        first = min(first, named ? i : k);
    }
    return sum;
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

// The student's mass outside the teacher's places, against which the rest of the teacher's probability is held.  SO has it relative to
// the row's largest logit; where less than OUTSIDE_FAR is left of that, its terms leave fp32 one after the other (up to 2^20 of them below
// 2^-126) while its logarithm is an ordinary number, so it is summed again relative to the largest logit outside.  (0: all of them are masked,
// nothing to sum.)
static constexpr float OUTSIDE_FAR = 0x1p-64f;
static constexpr int OUTSIDE_WORDS = 512;      // marks of 16384 places, for the kernels that have no marks of the whole row
struct Outside {
    bool apart = false;        // summed again: sum of exp((z - top)/T) over the places outside
    float top = 0.f, sum = 0.f;
};
__device__ __forceinline__ bool outside_far(const float4 &s, double rest) { return rest > 0.0 && s.w > 0.f && s.w < OUTSIDE_FAR && s.y > 0.f; }

// Two passes over the row, which is in the caches; every thread of the block calls it.  bits: marks of the teacher's places, `words` of
// them at a time.  Rare (students that put next to nothing outside, vocabularies masked with finite numbers): loss and gradient of 2048 rows
// of 131072 bf16, all of them such, 446 us against 239; of 16 rows of 262144 fp32, which a block each walks alone, 400 against 25.
template <int DT, int BLOCK>
__device__ __forceinline__ Outside outside_of(const Row<DT> &row, int place, const Scales &q, unsigned *bits, int words, float *fpart)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    const int tid = threadIdx.x, chunk = words * 32 / VEC;
    Outside o;
    o.apart = true;
    o.top = -INFINITY;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        float run = pass == 0 ? -INFINITY : 0.f;
#pragma unroll 1
        for (int s0 = 0; s0 < row.slots; s0 += chunk) {
            const int s1 = min(s0 + chunk, row.slots);
            __syncthreads();                            // everyone is done with the marks before these
            mark_places(bits, words, s0 * VEC, place, row.shift, BLOCK);
#pragma unroll 1
            for (int s = s0 + tid; s < s1; s += DEEP * BLOCK) {
                uint4 v[DEEP];
#pragma unroll
                for (int i = 0; i < DEEP; ++i) v[i] = s + i * BLOCK < s1 ? row.load(s + i * BLOCK) : Row<DT>::empty();
#pragma unroll
                for (int i = 0; i < DEEP; ++i) {
                    const unsigned skip = s + i * BLOCK < s1 ? marks_of<VEC>(bits, s + i * BLOCK - s0) : 0u;
                    float x[VEC];
                    Row<DT>::Type::unpack(v[i], x);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float here = skip >> j & 1 ? -INFINITY : x[j];
                        run = pass == 0 ? fmaxf(run, here) : run + exp2_fast((here - o.top) * q.c);
                    }
                }
            }
        }
        if (pass == 0) o.top = block_max<BLOCK>(run, fpart);
        else o.sum = block_sum<BLOCK>(run, fpart);
        if (o.top == -INFINITY) break;                  // uniform
    }
    return o;
}

// Whether a slot holds anything but -inf outside the teacher's places, which `skip` marks
template <int DT> __device__ __forceinline__ bool unmasked(const uint4 &raw, unsigned skip)
{
    const uint4 masked = Row<DT>::empty();
    unsigned d[4] = {raw.x ^ masked.x, raw.y ^ masked.y, raw.z ^ masked.z, raw.w ^ masked.w};
    if (skip) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (Row<DT>::VEC == 4) d[i] = skip >> i & 1 ? 0 : d[i];
            else d[i] &= (skip >> 2 * i & 1 ? 0 : 0xffffu) | (skip >> (2 * i + 1) & 1 ? 0 : 0xffff0000u);
        }
    }
    return (d[0] | d[1] | d[2] | d[3]) != 0;
}

// The row's loss from its sums (M, ST, S1, SO); every thread of the block calls it.
template <int BLOCK>
__device__ __forceinline__ void write_loss(const DistillArgs &a, size_t r, int place, float z_place, float z_label, bool padding,
                                           const float4 &s, const Outside &out, TeacherLds &lds)
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
    if (lds.rest > 0.0) {
        if (!out.apart && s.w > 0.f) kl += lds.rest * (log(lds.rest) - log((double)s.w) + log_st);
        if (out.apart && out.sum > 0.f) kl += lds.rest * (log(lds.rest) - (((double)out.top - (double)s.x) / T + log((double)out.sum)) + log_st);
    }
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
// The factors of a row's gradient: outside the places that the teacher or the label names it is fq e_j + f1 h_j, less
// far exp((z_j - top)/T) where the mass outside has a sum of its own.
struct Factors {
    double soft, up_hard, cover, outside, far;
    __device__ __forceinline__ Factors(const DistillArgs &a, size_t r, const TeacherLds &teacher, const float4 &s, const Outside &out)
    {
        const double up = (double)a.scale * (a.dloss ? (double)a.dloss[r] : 1.0);
        const double rest = (out.apart ? out.sum : s.w) > 0.f ? teacher.rest : 0.0;
        soft = up * (1.0 - (double)a.hard) * (double)a.temperature;
        up_hard = up * (double)a.hard;
        cover = teacher.mass + rest;
        outside = rest > 0.0 && !out.apart ? cover - rest * (double)s.y / (double)s.w : cover;
        far = rest > 0.0 && out.apart ? soft * rest / (double)out.sum : 0.0;
    }
};
template <int VEC> struct Slope {
    float fq, f1, far, top;
    Reference<VEC> at;
    bool none;                 // nothing to learn: the gradient is 0
    bool apart;                // a row of large logits, or a mass outside with a sum of its own: its elements go through of_apart()
    __device__ __forceinline__ Slope(const DistillArgs &a, size_t r, const TeacherLds &teacher, bool padding, const float4 &s, const Outside &out, const Scales &q)
        : at(uniform(s.x), q)
    {
        none = padding || uniform(s.y) == 0.f;
        apart = at.by_difference() || out.apart;
        const Factors f(a, r, teacher, s, out);
        fq = uniform((float)(f.soft * f.outside / (double)s.y) * exp2_fast(apart ? 0.f : -at.lost));
        f1 = a.hard > 0.f ? uniform((float)(f.up_hard / (double)s.z) * exp2_fast(apart ? 0.f : -at.lost1)) : 0.f;
        far = uniform((float)f.far);
        top = uniform(out.top);
    }
    __device__ __forceinline__ void of_apart(float (&x)[VEC], const Scales &q) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float d = x[i] - at.ref;
            const float beyond = far != 0.f ? far * exp2_fast((x[i] - top) * q.c) : 0.f;       // the teacher's own places are stored anew
            x[i] = fmaf(f1, exp2_fast(d * q.c1), fq * exp2_fast(d * q.c)) - beyond;
        }
    }
    template <int HARD> __device__ __forceinline__ void of(float (&x)[VEC]) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float e = at.soft(x[i]);
            if constexpr (HARD == HARD_PLAIN) x[i] = (fq + f1) * e;          // h = e
            else if constexpr (HARD == HARD_SQUARE) x[i] = e * fmaf(f1, e, fq);
            else x[i] = fmaf(f1, at.hard(x[i]), fq * e);
        }
    }
};

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
    __device__ __forceinline__ void put(int j, float d) const { row[j] = Type::narrow(d); }
    // 0 for slots first + thread, first + thread + block, ... below last
    __device__ __forceinline__ void clear(int last, int block, int first = 0) const
    {
        const float zero[VEC] = {};
        for (int s = first + threadIdx.x; s < last; s += block) store(s, zero, s * VEC >= shift && (s + 1) * VEC <= shift + V);
    }
};

// The gradient of slots [s0, s1) where Slope asks for the careful way.
template <int DT, int BLOCK>
__device__ __forceinline__ void put_apart(const Row<DT> &row, const GradRow<DT> &out, const Slope<Row<DT>::VEC> &g, const Scales &q, int s0, int s1)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 2;
#pragma unroll 1
    for (int s = s0 + (int)threadIdx.x; s < s1; s += DEEP * BLOCK) {
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if (s + i * BLOCK < s1) v[i] = row.load(s + i * BLOCK);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            if (s + i * BLOCK >= s1) break;
            float x[VEC];
            Row<DT>::Type::unpack(v[i], x);
            g.of_apart(x, q);
            out.store(s + i * BLOCK, x, row.full(s + i * BLOCK));
        }
    }
}

// The places that the teacher or the label names, within elements [j0, j1) (j0 may lie before the row): each once, by the
// first slot that names it, after a barrier behind the stores of all others.
template <int DT>
__device__ __forceinline__ void name_places(const DistillArgs &a, size_t r, const GradRow<DT> &out, int place, float z_place, int label,
                                            float z_label, const float4 &s, const Outside &outside, const TeacherLds &lds, int j0, int j1)
{
    const bool labelled = a.hard > 0.f;
    int at = -1;
    double target = 0.0;
    if (place >= max(j0, 0) && place < j1) {
        at = place;
        target = lds.p[threadIdx.x];
        if (slots_of(lds.index, a.k, place) > 1) {      // named again: the first slot adds all up
            int first;
            target = mass_of(lds.index, lds.p, a.k, place, first);
            if (first < (int)threadIdx.x) at = -1;
        }
    }
    const Factors f(a, r, lds, s, outside);
    auto name = [&](int j, float z, bool top, double goal) {
        const double x = (double)z - (double)s.x;
        double d = f.soft * ((top ? f.cover : f.outside) * exp(x / (double)a.temperature) / (double)s.y - goal);
        if (!top && f.far != 0.0) d -= f.far * exp(((double)z - (double)outside.top) / (double)a.temperature);
        if (f.up_hard != 0.0) d += f.up_hard * (exp(x) / (double)s.z - (labelled && j == label ? 1.0 : 0.0));
        out.put(j, (float)d);
    };
    const bool alone = labelled && threadIdx.x == blockDim.x - 1 && label >= j0 && label < j1 && slots_of(lds.index, a.k, label) == 0;    // a label that no slot names
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        const int j = turn == 0 ? at : alone ? label : -1;
        if (j >= 0) name(j, turn == 0 ? z_place : z_label, turn == 0, target);
        target = 0.0;
    }
}

// ---- loss, and gradient with GRAD, of whole rows, a block each -----------------------------------------------------
// The first NV * BLOCK slots of a row are requested at once and stay in registers between the two passes over it; what is
// longer is read again, from the last-level cache while no more rows are under way than it holds.  Gradients are stored past the
// caches (nobody reads them here).  Measured: 2048 x 131072 bf16, loss and gradient, 232 us = 4.6 TB/s of what has to move, with
// the vector ALUs 50 % busy (a copy of that size by the library takes 203); 777 x 50001 fp16 43 us = 3.6 TB/s (its rows start at
// odd addresses; copy 31).  A row of 2048 logits costs its block more in the teacher's numbers than in the row: 16384 x 2048
// bf16, k = 64, 117 us against 20 for a copy (both on one set of inputs, which the last-level cache holds).
template <int DT, int BLOCK, int NV, bool TAIL, int HARD, bool GRAD>
__global__ __launch_bounds__(BLOCK, 4) void distill_rows_kernel(DistillArgs a)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    static_assert(NV % DEEP == 0, "slots are looked at in groups");
    using Type = LogitType<DT>;
    extern __shared__ unsigned in_top[];
    __shared__ TeacherLds lds;
    __shared__ float4 part[BLOCK / 64];
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const Scales q(a.temperature, a.hard > 0.f);
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;
    Slot slot;
    slot.load(a, r);

    // full slots [f0, f1): thread t has f0 + t + i * BLOCK; threads 0 and 1 have the partial slots at the row's ends.  Loops run
    // for whole wavefronts (those whose first slot is there); lanes behind the end hold empty slots.
    const int f0 = row.first_full(), f1 = row.end_full();
    const int first = f0 + __builtin_amdgcn_readfirstlane(tid & ~63);
    uint4 v[NV], edge = Row<DT>::empty();
    int edge_slot = -1;
    if (tid == 0 && row.shift) edge_slot = 0;
    if (tid == 1 && row.slots > f1 && (row.slots > 1 || !row.shift)) edge_slot = row.slots - 1;
    if (!padding) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int s = f0 + tid + i * BLOCK;
            if (first + i * BLOCK < f1) v[i] = s < f1 ? row.load_once(s) : Row<DT>::empty();
        }
        if (edge_slot >= 0) edge = row.load(edge_slot);
    }
    const int place = read_teacher<BLOCK, TAIL>(a, r, slot, lds);
    float4 sums = make_float4(0.f, 0.f, 0.f, 0.f);
    float z_place = 0.f, z_label = 0.f;
    if (!padding) {                                     // uniform
        if (place >= 0) z_place = row.load_one(place);
        z_label = row.load_one(label);
        if constexpr (TAIL) mark_places(in_top, (row.slots * VEC + 31) / 32, 0, place, row.shift, BLOCK);
        RowSums<VEC, TAIL, HARD> acc(q);
        auto add = [&](const uint4 &raw, int s) {
            float x[VEC];
            Type::unpack(raw, x);
            acc.add(x, TAIL ? marks_of<VEC>(in_top, s) : 0u);
        };
        auto look = [&](const uint4 &raw, int s) { acc.some = acc.some || unmasked<DT>(raw, marks_of<VEC>(in_top, s)); };
        if (tid < 64) {
            add(edge, max(edge_slot, 0));
            acc.until_settled([&] { look(edge, max(edge_slot, 0)); });
        }
#pragma unroll
        for (int i0 = 0; i0 < NV; i0 += DEEP) {
#pragma unroll
            for (int i = i0; i < i0 + DEEP; ++i)
                if (first + i * BLOCK < f1) add(v[i], min(f0 + tid + i * BLOCK, f1 - 1));
            acc.until_settled([&] {
#pragma unroll
                for (int i = i0; i < i0 + DEEP; ++i)
                    if (first + i * BLOCK < f1) look(v[i], min(f0 + tid + i * BLOCK, f1 - 1));
            });
        }
        for (int i0 = NV; first + i0 * BLOCK < f1; i0 += DEEP) {
            uint4 w[DEEP];
#pragma unroll
            for (int i = 0; i < DEEP; ++i) {
                const int s = f0 + tid + (i0 + i) * BLOCK;
                w[i] = s < f1 ? row.load_full(s) : Row<DT>::empty();
            }
#pragma unroll
            for (int i = 0; i < DEEP; ++i)
                if (first + (i0 + i) * BLOCK < f1) add(w[i], min(f0 + tid + (i0 + i) * BLOCK, f1 - 1));
            acc.until_settled([&] {
#pragma unroll
                for (int i = 0; i < DEEP; ++i)
                    if (first + (i0 + i) * BLOCK < f1) look(w[i], min(f0 + tid + (i0 + i) * BLOCK, f1 - 1));
            });
        }
        sums = acc.template combine<BLOCK>(part);
    }
    Outside outside;
    if constexpr (TAIL)
        if (!padding && outside_far(sums, lds.rest)) outside = outside_of<DT, BLOCK>(row, place, q, in_top, (row.slots * VEC + 31) / 32, lds.fpart);
    if constexpr (GRAD) {
        const GradRow<DT> out(a, r, row);
        const Slope<VEC> g(a, r, lds, padding, sums, outside, q);
        auto put = [&](const uint4 &raw, int s, bool full) {
            float x[VEC];
            Type::unpack(raw, x);
            g.template of<HARD>(x);
            out.store(s, x, full);
        };
        if (g.none) {                                   // uniform
            out.clear(row.slots, BLOCK);
        } else if (g.apart) {                           // uniform, and rare: the row is read again
            put_apart<DT, BLOCK>(row, out, g, q, 0, row.slots);
        } else {
            for (int s0 = f0 + tid + NV * BLOCK; s0 < f1; s0 += DEEP * BLOCK) {
                uint4 w[DEEP];
#pragma unroll
                for (int i = 0; i < DEEP; ++i)
                    if (s0 + i * BLOCK < f1) w[i] = row.load_full(s0 + i * BLOCK);
#pragma unroll
                for (int i = 0; i < DEEP; ++i)
                    if (s0 + i * BLOCK < f1) put(w[i], s0 + i * BLOCK, true);
            }
            if (edge_slot >= 0) put(edge, edge_slot, false);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (f0 + tid + i * BLOCK < f1) put(v[i], f0 + tid + i * BLOCK, true);
        }
        write_loss<BLOCK>(a, r, place, z_place, z_label, padding, sums, outside, lds);       // its barriers stand between the stores above and below
        if (!g.none) name_places<DT>(a, r, out, place, z_place, label, z_label, sums, outside, lds, 0, a.V);
    } else {
        write_loss<BLOCK>(a, r, place, z_place, z_label, padding, sums, outside, lds);
    }
}

// ---- few rows: sums of parts of rows ----------------------------------------------------------------------------------
// A row by a block each would leave most of the chip idle: its parts are summed by blocks of their own, which leave four floats
// each (maximum and sums), and distill_join_kernel adds them in the order of the parts.  Bound: latency.  16 x 262144 fp32:
// 6.5 us, and 5.0 for the join, which waits for it; a block per row took 119 us in all.
template <int DT, int BLOCK, bool TAIL, int HARD>
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
    const Scales q(a.temperature, a.hard > 0.f);
    if (a.labels && (unsigned)a.labels[r] >= (unsigned)a.V) return;
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    if constexpr (TAIL) {
        int place = -1;
        if (tid < a.k) place = a.indices[r * a.k + tid];
        if ((unsigned)place >= (unsigned)a.V) place = -1;
        mark_places(in_top, (a.seg_slots * VEC + 31) / 32, s0 * VEC, place, row.shift, BLOCK);
    }
    RowSums<VEC, TAIL, HARD> acc(q);
    auto add = [&](const uint4 &raw, int s) {
        float x[VEC];
        Type::unpack(raw, x);
        acc.add(x, TAIL ? marks_of<VEC>(in_top, s - s0) : 0u);
    };
    auto look = [&](const uint4 &raw, int s) { acc.some = acc.some || unmasked<DT>(raw, marks_of<VEC>(in_top, s - s0)); };
    const int lead = __builtin_amdgcn_readfirstlane(tid & ~63);
    int s = s0 + tid;
    for (; s - tid + DEEP * BLOCK <= s1; s += DEEP * BLOCK) {      // uniform
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) v[i] = row.load(s + i * BLOCK);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) add(v[i], s + i * BLOCK);
        acc.until_settled([&] {
#pragma unroll
            for (int i = 0; i < DEEP; ++i) look(v[i], s + i * BLOCK);
        });
    }
    for (; s - tid + lead < s1; s += BLOCK) {           // whole wavefronts
        const uint4 v = s < s1 ? row.load(s) : Row<DT>::empty();
        add(v, min(s, s1 - 1));
        acc.until_settled([&] { look(v, min(s, s1 - 1)); });
    }
    const float4 sums = acc.template combine<BLOCK>(part);
    if (tid == 0) a.partial[r * a.segments + seg] = sums;
}

// ---- the losses of rows whose parts were summed apart ----------------------------------------------------------------
template <int DT, bool TAIL>
__global__ __launch_bounds__(256) void distill_join_kernel(DistillArgs a)
{
    __shared__ TeacherLds lds;
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const Scales q(a.temperature, a.hard > 0.f);
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;
    Slot slot;
    slot.load(a, r);
    const int place = read_teacher<256, TAIL>(a, r, slot, lds);
    float4 sums = make_float4(0.f, 0.f, 0.f, 0.f);
    float z_place = 0.f, z_label = 0.f;
    if (!padding) {
        if (place >= 0) z_place = row.load_one(place);
        if (threadIdx.x == 0) z_label = row.load_one(label);
        // a part per thread, in a fixed order
        float4 own = make_float4(-INFINITY, 0.f, 0.f, 0.f);
        for (int i = threadIdx.x; i < a.segments; i += 256) {
            const float4 p = a.partial[r * a.segments + i];
            const float4 w = own;
            own = make_float4(fmaxf(w.x, p.x), 0.f, 0.f, 0.f);
            RowSums<4, TAIL, HARD_EXP>::join(own, w, q);
            RowSums<4, TAIL, HARD_EXP>::join(own, p, q);
        }
        sums.x = block_max<256>(own.x, lds.fpart);
        RowSums<4, TAIL, HARD_EXP>::join(sums, own, q);
        sums.y = block_sum<256>(sums.y, lds.fpart);
        sums.z = block_sum<256>(sums.z, lds.fpart);
        sums.w = block_sum<256>(sums.w, lds.fpart);
    }
    Outside outside;
    if constexpr (TAIL) {
        __shared__ unsigned bits[OUTSIDE_WORDS];
        if (!padding && outside_far(sums, lds.rest)) outside = outside_of<DT, 256>(row, place, q, bits, OUTSIDE_WORDS, lds.fpart);
    }
    write_loss<256>(a, r, place, z_place, z_label, padding, sums, outside, lds);
}

// ---- backward: gradients of parts of rows ----------------------------------------------------------------------------
// The forward pass left a row's sums, so that this is one pass with one exponential a logit (two where hard asks for another).
// Bound: HBM, and one wave of blocks that ask for their first logits when the teacher's numbers are done.  1024 x 32000 bf16: 32.8 us = 4.0 TB/s.
template <int DT, int BLOCK, bool TAIL, int HARD>
__global__ __launch_bounds__(BLOCK) void distill_grad_kernel(DistillArgs a)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    using Type = LogitType<DT>;
    __shared__ TeacherLds lds;
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const Scales q(a.temperature, a.hard > 0.f);
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    Slot slot;
    slot.load(a, r);
    const int place = read_teacher<BLOCK, TAIL>(a, r, slot, lds);
    const float4 sums = reinterpret_cast<const float4 *>(a.state)[r];
    Outside outside;
    if constexpr (TAIL) {
        __shared__ unsigned bits[OUTSIDE_WORDS];
        if (!padding && outside_far(sums, lds.rest)) outside = outside_of<DT, BLOCK>(row, place, q, bits, OUTSIDE_WORDS, lds.fpart);
    }
    const Slope<VEC> g(a, r, lds, padding, sums, outside, q);
    const GradRow<DT> out(a, r, row);
    auto put = [&](const uint4 &raw, int s) {
        float x[VEC];
        Type::unpack(raw, x);
        g.template of<HARD>(x);
        out.store(s, x, row.full(s));
    };
    int s = s0 + tid;
    if (g.none) {
        out.clear(s1, BLOCK, s0);
        return;
    }
    const float z_place = place >= 0 ? row.load_one(place) : 0.f, z_label = row.load_one(label);
    if (g.apart) {                                      // uniform, and rare
        put_apart<DT, BLOCK>(row, out, g, q, s0, s1);
        s = s1;
    }
    for (; s - tid + DEEP * BLOCK <= s1; s += DEEP * BLOCK) {
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) v[i] = row.full(s + i * BLOCK) ? row.load_once(s + i * BLOCK) : row.load(s + i * BLOCK);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) put(v[i], s + i * BLOCK);
    }
    for (; s < s1; s += BLOCK) put(row.load(s), s);
    __syncthreads();
    name_places<DT>(a, r, out, place, z_place, label, z_label, sums, outside, lds, s0 * VEC - row.shift, s1 * VEC - row.shift);
}

// ---- short rows: a wavefront each, all three calls --------------------------------------------------------------------
// Rows of at most 64 * NQ logits sit in a wavefront's registers, element lane + 64 q in x[q]; maximum and sums are shuffles,
// and nothing waits for other wavefronts.  LDS holds the teacher's slots and, for every element, its target (-1: not one
// of the teacher's places).  Bound: latency (one trip to memory, two chains of 64-bit exponentials and logarithms).
// Measured: 2048 x 100 fp32 7.6 us, of which a launch that does nothing is some 2.  Beyond 1024 logits a block a row is faster
// (16384 x 2040 bf16: 136 us, 202 with 32 registers a lane here).
template <int DT, int NQ, bool TAIL, int MODE>
__global__ __launch_bounds__(256, 4) void distill_short_kernel(DistillArgs a)
{
    using Type = LogitType<DT>;
    constexpr int SLOTS = LOGITS_MAX_TOP / 64;
    __shared__ __attribute__((aligned(16))) int all_index[4][LOGITS_MAX_TOP];
    __shared__ double all_p[4][LOGITS_MAX_TOP];
    __shared__ float all_target[4][NQ * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t r = (size_t)blockIdx.x * 4 + wave;
    if (r >= a.rows) return;                            // wavefronts of a block have nothing in common
    int *index = all_index[wave];
    double *probability = all_p[wave];
    float *target = all_target[wave];
    // LDS accesses of one wavefront are executed in order: only the compiler has to keep them so
    auto in_order = []() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); };

    const Row<DT> row(a.logits, r, a.ld, a.V);
    const Scales q(a.temperature, a.hard > 0.f);
    const double T = (double)a.temperature;
    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V, hard = a.hard > 0.f;
    int place[SLOTS];
    float value[SLOTS], z_place[SLOTS], x[NQ];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        const int i = lane + 64 * j;
        place[j] = i < a.k ? a.indices[r * a.k + i] : -1;
        value[j] = i < a.k ? a.values[r * a.k + i] : 0.f;
    }
    const float lse_given = TAIL ? a.teacher_lse[r] : 0.f;
    auto logit_at = [&](int j) {
        float z = row.load_one(j);
        if constexpr (DT == EASGD_F32)                  // logits that come as partial sums: added in ascending order
            for (int s = 1; s < a.parts; ++s) z += row.base[row.shift + j + s * a.part_stride];
        return z;
    };
#pragma unroll
    for (int c = 0; c < NQ; ++c) x[c] = lane + 64 * c < a.V && !padding ? logit_at(lane + 64 * c) : -INFINITY;
    float z_label = 0.f;
#pragma unroll
    for (int c = 0; c < NQ; ++c) z_label = lane + 64 * c == label ? x[c] : z_label;
    z_label = wave_only(z_label);

    // the teacher
    double log_p[SLOTS], p[SLOTS], mass = 0.0;
    float top = -INFINITY;
    bool live[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        if ((unsigned)place[j] >= (unsigned)a.V) place[j] = -1;
        live[j] = place[j] >= 0 && value[j] != -INFINITY && !(TAIL && lse_given == -INFINITY);       // as in read_teacher
        log_p[j] = -(double)INFINITY;
        if (live[j]) top = fmaxf(top, value[j]);
    }
    if constexpr (TAIL) {
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
            if (live[j]) log_p[j] = (double)value[j] / T - (double)lse_given;
    } else {
        top = wave_max(top);
        double total = 0.0;
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            if (live[j]) {
                log_p[j] = ((double)value[j] - (double)top) / T;
                total += exp(log_p[j]);
            }
        }
        const double log_total = log(wave_sum(total));
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
            if (live[j]) log_p[j] -= log_total;
    }
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        const int i = lane + 64 * j;
        p[j] = 0.0;
        if (64 * j < a.k) {
            p[j] = place[j] >= 0 ? exp(log_p[j]) : 0.0;
            index[i] = place[j];
            probability[i] = p[j];
        }
        mass += p[j];
    }
    mass = wave_sum(mass);
    double rest = TAIL && mass < 1.0 ? 1.0 - mass : 0.0;
#pragma unroll
    for (int c = 0; c < NQ; ++c) target[lane + 64 * c] = -1.f;
    in_order();
    // a place that is named again: its first slot adds all up, in their order.  A lane's slots go through the teacher's together.
    int named[SLOTS] = {}, first[SLOTS];
    double sum[SLOTS];
#pragma unroll 2
    for (int i = 0; i < a.k; i += 4) {
        const int4 q = *reinterpret_cast<const int4 *>(index + i);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) named[j] += (q.x == place[j]) + (q.y == place[j]) + (q.z == place[j]) + (q.w == place[j]);
    }
    bool again = false;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        again |= place[j] >= 0 && named[j] > 1;
        first[j] = lane + 64 * j;
        sum[j] = p[j];
    }
    if (__any(again)) {
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) sum[j] = 0.0;
#pragma unroll 4
        for (int i = 0; i < a.k; ++i) {
            const int here = index[i];
            const double mass_here = probability[i];
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                const bool is = here == place[j];
                sum[j] += is ? mass_here : 0.0;
                first[j] = min(first[j], is ? i : LOGITS_MAX_TOP);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < SLOTS; ++j)
        if (place[j] >= 0 && first[j] == lane + 64 * j) target[place[j]] = (float)sum[j];
    in_order();

    // maximum and sums
    float e[NQ], h[NQ], t[NQ];
    float4 s;
    if constexpr (MODE & DISTILL_LOSS) {
        float m = x[0];
#pragma unroll
        for (int c = 1; c < NQ; ++c) m = fmaxf(m, x[c]);
        s.x = wave_max(m);
    } else s = reinterpret_cast<const float4 *>(a.state)[r];
    const float m = s.x == -INFINITY ? 0.f : s.x;
    float st = 0.f, s1 = 0.f, so = 0.f;
    bool some = false;
#pragma unroll
    for (int c = 0; c < NQ; ++c) {
        t[c] = target[lane + 64 * c];
        if constexpr (TAIL && (MODE & DISTILL_LOSS)) some = some || (!(t[c] >= 0.f) && x[c] > -INFINITY);
        e[c] = exp2_fast((x[c] - m) * q.c);
        h[c] = !hard ? 0.f : a.temperature == 1.f ? e[c] : exp2_fast((x[c] - m) * q.c1);
        st += e[c];
        s1 += h[c];
        so += t[c] >= 0.f ? 0.f : e[c];
    }
    if constexpr (MODE & DISTILL_LOSS) {
        s.y = wave_sum(st);
        s.z = hard ? wave_sum(s1) : 0.f;
        s.w = TAIL ? wave_sum(so) : 0.f;
        if (TAIL && s.w == 0.f && __any(some)) s.w = OUTSIDE_TINY;
    }
    const bool none = padding || s.y == 0.f;
    Outside outside;
    if constexpr (TAIL) {
        if (__any(!padding && outside_far(s, rest))) {  // uniform; the row is read again: registers would cost every row
            float top = -INFINITY, sum = 0.f;
#pragma unroll 1
            for (int j = lane; j < a.V; j += 64) top = fmaxf(top, target[j] >= 0.f ? -INFINITY : logit_at(j));
            top = wave_max(top);
            if (top > -INFINITY) {
#pragma unroll 1
                for (int j = lane; j < a.V; j += 64) sum += target[j] >= 0.f ? 0.f : exp2_fast((logit_at(j) - top) * q.c);
            }
            outside.apart = true;
            outside.top = top;
            outside.sum = wave_sum(sum);
        }
    }
    if (!((outside.apart ? outside.sum : s.w) > 0.f)) rest = 0.0;

    if constexpr (MODE & DISTILL_LOSS) {
        const double log_st = log((double)s.y);
        double kl = 0.0;
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            if (64 * j >= a.k) break;
            z_place[j] = 0.f;
            if (!none && place[j] >= 0) z_place[j] = logit_at(place[j]);
            if (!none && p[j] > 0.0) kl += p[j] * (log_p[j] - (((double)z_place[j] - (double)s.x) / T - log_st));
            if (isnan(p[j])) kl += p[j];
        }
        kl = wave_sum(kl);
        if (lane == 0) {
            if (rest > 0.0) {
                const double log_so = outside.apart ? ((double)outside.top - (double)s.x) / T + log((double)outside.sum) : log((double)s.w);
                kl += rest * (log(rest) - log_so + log_st);
            }
            double loss = 0.0;
            if (!none) {
                if (a.hard < 1.f) loss = (1.0 - (double)a.hard) * T * T * kl;
                if (hard) loss += (double)a.hard * (((double)s.x - (double)z_label) + log((double)s.z));
                if (isnan(s.y)) loss = NAN;
            }
            a.loss[r] = (float)loss;
            if (a.state) reinterpret_cast<float4 *>(a.state)[r] = padding ? make_float4(0.f, 0.f, 0.f, 0.f) : s;
        }
    }
    if constexpr (MODE & DISTILL_GRAD) {
        const double up = (double)a.scale * (a.dloss ? (double)a.dloss[r] : 1.0), soft = up * (1.0 - (double)a.hard) * T;
        const double cover = mass + rest, all_out = rest > 0.0 && !outside.apart ? cover - rest * (double)s.y / (double)s.w : cover;
        const float f_in = (float)(soft * cover / (double)s.y), f_out = (float)(soft * all_out / (double)s.y), f_t = (float)soft;
        const float far = rest > 0.0 && outside.apart ? (float)(soft * rest / (double)outside.sum) : 0.f;
        const float f1 = hard ? (float)(up * (double)a.hard / (double)s.z) : 0.f, f_y = (float)(up * (double)a.hard);
        const Row<DT> out(a.dlogits, r, a.dld, a.V);
        auto put = [&](int j, float target_j, float e_j, float h_j, float beyond) {
            const bool in = target_j >= 0.f;
            float d = fmaf(f1, h_j, (in ? f_in : f_out) * e_j);
            if (in) d = fmaf(-f_t, target_j, d);
            else d -= beyond;
            if (hard && j == label) d -= f_y;
            out.base[out.shift + j] = Type::narrow(none ? 0.f : d);
        };
        if (TAIL && __any(far != 0.f)) {                // uniform, and rare: the row is read again
#pragma unroll 1
            for (int j = lane; j < a.V; j += 64) {
                const float z = logit_at(j), e_j = exp2_fast((z - m) * q.c);
                put(j, target[j], e_j, a.temperature == 1.f ? e_j : exp2_fast((z - m) * q.c1), far * exp2_fast((z - outside.top) * q.c));
            }
            return;
        }
#pragma unroll
        for (int c = 0; c < NQ; ++c)
            if (lane + 64 * c < a.V) put(lane + 64 * c, t[c], e[c], h[c], 0.f);
    }
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

int check_teacher(const char *name, const TeacherGiven &t, bool rows)
{
    if (t.k < 1 || t.k > LOGITS_MAX_TOP) return fail(EASGD_EINVAL, "%s: k must be in [1, %d], got %d", name, LOGITS_MAX_TOP, t.k);
    if (int rc = check_temperature(name, t.temperature)) return rc;
    if (!(t.hard >= 0.f && t.hard <= 1.f)) return fail(EASGD_EINVAL, "%s: hard must be in [0, 1], got %g", name, (double)t.hard);
    if (!t.labels && t.hard != 0.f) return fail(EASGD_EINVAL, "%s: hard = %g needs labels", name, (double)t.hard);
    if (rows && (!t.indices || !t.values)) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(t.indices, 4) || !aligned_to(t.values, 4) || !aligned_to(t.lse, 4) || !aligned_to(t.labels, 4))
        return fail(EASGD_EINVAL, "%s: indices, values, teacher_lse, labels must be 4-byte aligned", name);
    return EASGD_OK;
}

static int check_distill(const DistillCall &q, int mode)
{
    const DistillArgs &a = q.a;
    if (int rc = check_logits(q.name, a.logits, q.dtype, q.rows, a.V, a.ld)) return rc;
    if (int rc = check_teacher(q.name, {a.indices, a.values, a.teacher_lse, a.k, a.labels, a.temperature, a.hard}, q.rows > 0)) return rc;
    if (q.rows > 0 && (((mode & DISTILL_LOSS) && !a.loss) || (mode == DISTILL_GRAD && !a.state) || ((mode & DISTILL_GRAD) && !a.dlogits)))
        return fail(EASGD_EINVAL, "%s: NULL pointer", q.name);
    if (!aligned_to(a.loss, 4) || !aligned_to(a.dloss, 4)) return fail(EASGD_EINVAL, "%s: loss, dloss must be 4-byte aligned", q.name);
    if (!aligned16(a.state)) return fail(EASGD_EINVAL, "%s: state must be 16-byte aligned", q.name);
    if (mode & DISTILL_GRAD) {
        if (!std::isfinite(a.scale)) return fail(EASGD_EINVAL, "%s: scale must be finite", q.name);
        if (a.dld < (size_t)a.V) return fail(EASGD_EINVAL, "%s: dld (%zu) < V (%d)", q.name, a.dld, a.V);
        if (q.rows > 1 && a.dld > ((size_t)1 << 60) / q.rows) return fail(EASGD_ERANGE, "%s: rows * dld too large", q.name);
        if (!aligned_to(a.dlogits, dtype_bytes(q.dtype))) return fail(EASGD_EINVAL, "%s: dlogits must be aligned to its elements (%zu bytes)", q.name, dtype_bytes(q.dtype));
    }
    return EASGD_OK;
}

// Whether a row of logits and one of dlogits share memory: blocks read a row, or parts of others, while they store.  Rows that
// alternate (the two halves of wider rows, say) share none; at two strides the whole ranges have to be apart.
static bool rows_overlap(const DistillArgs &a, size_t rows, size_t size)
{
    const uintptr_t in = reinterpret_cast<uintptr_t>(a.logits), out = reinterpret_cast<uintptr_t>(a.dlogits);
    const size_t row = (size_t)a.V * size;
    if (in + (rows - 1) * a.ld * size + row <= out || out + (rows - 1) * a.dld * size + row <= in) return false;
    if (rows == 1 || a.ld != a.dld) return true;
    const size_t pitch = a.ld * size, apart = in < out ? (out - in) % pitch : (in - out) % pitch;
    return apart < row || pitch - apart < row;
}

// Into how many parts rows are cut: enough blocks to fill the chip, and at least 1024 slots (four per thread) a part.
static constexpr int SPLIT_ROWS = 256, SPLIT_BLOCKS = 1024, SPLIT_SLOTS = 1024;
static int segments_of(size_t rows, int slots)
{
    if (rows >= SPLIT_ROWS || slots < 2 * SPLIT_SLOTS) return 1;
    const int want = (int)((SPLIT_BLOCKS + rows - 1) / rows), most = slots / SPLIT_SLOTS;
    return want < most ? want : most;
}
static void set_segments(DistillArgs &a, int segments, int slots)
{
    a.segments = segments;
    a.seg_slots = ((slots + segments - 1) / segments + 7) / 8 * 8;      // a multiple of 8: parts of the bit map begin at whole words
}

// calls f with the kind of the hard exponentials and whether there is a teacher's log-sum-exp as constants
template <typename F> static void by_kind(const DistillArgs &a, F f)
{
    auto with = [&](auto tail) {
        if (!(a.hard > 0.f) || a.temperature == 1.f) f(tail, std::integral_constant<int, HARD_PLAIN>{});
        else if (a.temperature == 2.f) f(tail, std::integral_constant<int, HARD_SQUARE>{});
        else f(tail, std::integral_constant<int, HARD_EXP>{});
    };
    if (a.teacher_lse) with(std::true_type{});
    else with(std::false_type{});
}

template <int DT> static void launch_sums(const DistillArgs &a, hipStream_t s)
{
    const size_t bits = a.teacher_lse ? ((size_t)a.seg_slots * LogitType<DT>::VEC + 31) / 32 * 4 : 0;
    by_kind(a, [&](auto tail, auto hard) {
        EASGD_LAUNCH((distill_sums_kernel<DT, 256, decltype(tail)::value, decltype(hard)::value>), dim3((unsigned)(a.rows * a.segments)), dim3(256), bits, s, a);
    });
    if (a.teacher_lse) EASGD_LAUNCH((distill_join_kernel<DT, true>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
    else EASGD_LAUNCH((distill_join_kernel<DT, false>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
}

template <int DT> static void launch_grad(const DistillArgs &a, hipStream_t s)
{
    by_kind(a, [&](auto tail, auto hard) {
        EASGD_LAUNCH((distill_grad_kernel<DT, 256, decltype(tail)::value, decltype(hard)::value>), dim3((unsigned)(a.rows * a.segments)), dim3(256), 0, s, a);
    });
}

template <int DT, int BLOCK, int NV, bool GRAD> static void launch_block(const DistillArgs &a, hipStream_t s)
{
    constexpr int VEC = LogitType<DT>::VEC;
    const size_t bits = a.teacher_lse ? ((size_t)a.V + VEC - 1 + 31) / 32 * 4 + 4 : 0;
    by_kind(a, [&](auto tail, auto hard) {
        EASGD_LAUNCH((distill_rows_kernel<DT, BLOCK, NV, decltype(tail)::value, decltype(hard)::value, GRAD>), dim3((unsigned)a.rows), dim3(BLOCK), bits, s, a);
    });
}

// The block's size goes by the row's length alone, so that the forward pass adds in the same order with and without the gradient.
// Loss and gradient in us, blocks of 256 threads that hold 4 slots a thread / 256 that hold 12 / 512 that hold 8:
//   4096 x 8192 bf16 54 / 60 / 62      4096 x 32000 bf16 122 / 116 / 117      777 x 50001 fp16 47 / 46.5 / 53
//   2048 x 65536 bf16 140 / 123 / 123  2048 x 131072 bf16 279 / 254 / 241
// Short rows want many blocks a compute unit (six against four); long ones few, whose rows the last-level cache (256 MB) holds
// between the two passes: 1024 rows under way of 256 KB are too many.
template <int DT, bool GRAD> static void launch_rows(const DistillArgs &a, int slots, hipStream_t s)
{
    if (slots <= 2048) launch_block<DT, 256, 4, GRAD>(a, s);
    else if (slots <= 8192 + 2) launch_block<DT, 256, 12, GRAD>(a, s);
    else launch_block<DT, 512, 8, GRAD>(a, s);
}

// Rows that a wavefront holds
static constexpr int SHORT_V = DISTILL_SHORT_V;

template <int DT, int NQ, int MODE> static void launch_short_nq(const DistillArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.rows + 3) / 4));
    if (a.teacher_lse) EASGD_LAUNCH((distill_short_kernel<DT, NQ, true, MODE>), grid, dim3(256), 0, s, a);
    else EASGD_LAUNCH((distill_short_kernel<DT, NQ, false, MODE>), grid, dim3(256), 0, s, a);
}
template <int DT, int MODE> static void launch_short(const DistillArgs &a, hipStream_t s)
{
    if (a.V <= 128) launch_short_nq<DT, 2, MODE>(a, s);
    else launch_short_nq<DT, SHORT_V / 64, MODE>(a, s);
}

void distill_logits(const float *logits, int parts, size_t part_stride, size_t rows, int classes, const TeacherGiven &t, float scale,
                    float *row_loss, float *dlogits, void *stream)
{
    const DistillArgs a = {logits, (size_t)classes, classes, t.k, t.indices, t.values, t.lse, t.labels, t.temperature, t.hard, row_loss, nullptr, nullptr,
                           scale, dlogits, (size_t)classes, rows, parts, part_stride, nullptr, 1, 0};
    launch_short<EASGD_F32, DISTILL_BOTH>(a, static_cast<hipStream_t>(stream));
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
        const size_t need = easgd_distill_workspace_bytes(q.rows, a.V, a.k);
        if (int rc = check_workspace(q.name, q.workspace, q.workspace_bytes, need)) return rc;
    }
    if ((MODE & DISTILL_GRAD) && q.rows && rows_overlap(a, q.rows, dtype_bytes(q.dtype))) return fail(EASGD_EINVAL, "%s: dlogits must not overlap logits", q.name);
    clear_error();
    if (q.rows == 0) return EASGD_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    a.partial = static_cast<float4 *>(q.workspace);
    by_dtype(q.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (a.V <= SHORT_V) launch_short<DT, MODE>(a, s);
        else if constexpr (MODE == DISTILL_GRAD) launch_grad<DT>(a, s);
        else if (segments == 1) launch_rows<DT, MODE == DISTILL_BOTH>(a, slots, s);
        else {
            if constexpr (MODE == DISTILL_BOTH) a.state = reinterpret_cast<float *>(a.partial + q.rows * segments);
            launch_sums<DT>(a, s);
            if constexpr (MODE == DISTILL_BOTH) launch_grad<DT>(a, s);
        }
    });
    return check_launch(q.name);
}

}  // namespace easgd

extern "C" {

size_t easgd_distill_workspace_bytes(size_t rows, int V, int)
{
    using namespace easgd;
    if (rows == 0 || rows > LOGITS_MAX_ROWS || V < 1 || V > LOGITS_MAX_V) return 0;
    const int most = segments_of(rows, most_slots(EASGD_F32, V)), least = segments_of(rows, most_slots(EASGD_BF16, V));
    return split_bytes(rows, most > least ? most : least);
}

int easgd_distill_loss(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                       const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, float *loss, float *state,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    easgd::DistillCall q = {"easgd_distill_loss", dtype, rows, {}, workspace, workspace_bytes};
    q.a = {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, loss, state, nullptr, 1.f, nullptr, 0, rows, 1, 0, nullptr, 1, 0};
    return easgd::launch_distill<easgd::DISTILL_LOSS>(q, stream);
}

int easgd_distill_grad(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                       const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, const float *state,
                       const float *dloss, float scale, void *dlogits, size_t dld, void *stream)
{
    easgd::DistillCall q = {"easgd_distill_grad", dtype, rows, {}, nullptr, 0};
    q.a = {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, nullptr, const_cast<float *>(state), dloss, scale, dlogits, dld, rows, 1, 0, nullptr, 1, 0};
    return easgd::launch_distill<easgd::DISTILL_GRAD>(q, stream);
}

int easgd_distill(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                  const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, float scale, float *loss,
                  void *dlogits, size_t dld, void *workspace, size_t workspace_bytes, void *stream)
{
    easgd::DistillCall q = {"easgd_distill", dtype, rows, {}, workspace, workspace_bytes};
    q.a = {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, loss, nullptr, nullptr, scale, dlogits, dld, rows, 1, 0, nullptr, 1, 0};
    return easgd::launch_distill<easgd::DISTILL_BOTH>(q, stream);
}

}  // extern "C"
