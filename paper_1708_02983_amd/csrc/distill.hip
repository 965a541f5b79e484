// Distillation from a teacher's top logits: the loss of every row and its gradient.
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
};

enum { DISTILL_LOSS = 1, DISTILL_GRAD = 2, DISTILL_BOTH = 3 };

// What a row's teacher asks for, in LDS: places, probabilities, and per place the sum over slots that name it.
struct Teacher {
    int index[LOGITS_MAX_TOP];             // -1: slot not used
    double log_p[LOGITS_MAX_TOP];
    double p[LOGITS_MAX_TOP];
};

template <int DT, int BLOCK, int MODE, bool TAIL>
__global__ __launch_bounds__(BLOCK) void distill_rows_kernel(DistillArgs a)
{
    constexpr int VEC = Row<DT>::VEC;
    using Type = LogitType<DT>;
    static_assert(BLOCK >= LOGITS_MAX_TOP, "one thread per slot of the teacher");
    extern __shared__ unsigned in_top[];               // TAIL: a bit per element of the row, by place on the 16-byte grid
    __shared__ Teacher t;
    __shared__ double dpart[BLOCK / 64];
    __shared__ float fpart[BLOCK / 64];
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const double T = (double)a.temperature;
    const float c = (float)(LOG2E / T), c1 = (float)LOG2E;

    const int label = a.labels ? a.labels[r] : 0;
    const bool padding = (unsigned)label >= (unsigned)a.V;
    const bool hard_row = a.labels != nullptr && a.hard > 0.f;

    // ---- the teacher ----
    int place = -1;
    double logit = -INFINITY;
    if (tid < a.k) {
        place = a.indices[r * a.k + tid];
        if ((unsigned)place >= (unsigned)a.V) place = -1;
        else logit = (double)a.values[r * a.k + tid] / T;
        t.index[tid] = place;
    }
    double lse_t;
    if constexpr (TAIL) lse_t = (double)a.teacher_lse[r];
    else {
        const float top = block_max<BLOCK>((float)logit, fpart);
        const double total = block_sum<BLOCK>(place >= 0 && top > -INFINITY ? exp(logit - (double)top) : 0.0, dpart);
        lse_t = (double)top + log(total);              // nothing but unused or masked slots: no probability anywhere
        if (!(top > -INFINITY)) lse_t = isnan(total) ? (double)NAN : 0.0;
    }
    const double log_p = logit - lse_t, p = place >= 0 ? exp(log_p) : 0.0;
    if (tid < a.k) t.p[tid] = p;
    const double mass = block_sum<BLOCK>(p, dpart);    // also: t is complete
    double rest = 0.0;
    if constexpr (TAIL) rest = mass < 1.0 ? 1.0 - mass : 0.0;

    // ---- forward: maximum and sums ----
    float M, ST, S1, SO;
    if constexpr (MODE & DISTILL_LOSS) {
        float m = -FLT_MAX, st = 0.f, s1 = 0.f, so = 0.f;
        if (!padding) {
            if constexpr (TAIL) {
                const int words = (row.slots * VEC + 31) / 32;
                for (int w = tid; w < words; w += BLOCK) in_top[w] = 0;
                __syncthreads();
                if (place >= 0) atomicOr(&in_top[(place + row.shift) >> 5], 1u << ((place + row.shift) & 31));
                __syncthreads();
            }
            for (int s = tid; s < row.slots; s += BLOCK) {
                float x[VEC];
                Type::unpack(row.load(s), x);
                float top = x[0];
#pragma unroll
                for (int i = 1; i < VEC; ++i) top = fmaxf(top, x[i]);
                if (top > m) {
                    const float f = exp2_fast((m - top) * c);
                    st *= f;
                    so *= f;
                    s1 *= exp2_fast((m - top) * c1);
                    m = top;
                }
                unsigned skip = 0;
                if constexpr (TAIL) skip = (in_top[s * VEC >> 5] >> (s * VEC & 31)) & ((1u << VEC) - 1);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float e = exp2_fast((x[i] - m) * c);
                    st += e;
                    if constexpr (TAIL) so += (skip >> i & 1) ? 0.f : e;
                    if (hard_row) s1 += exp2_fast((x[i] - m) * c1);
                }
            }
        }
        M = block_max<BLOCK>(m, fpart);
        const float f = exp2_fast((m - M) * c);
        ST = block_sum<BLOCK>(st * f, fpart);
        SO = TAIL ? block_sum<BLOCK>(so * f, fpart) : 0.f;
        S1 = hard_row ? block_sum<BLOCK>(s1 * exp2_fast((m - M) * c1), fpart) : 0.f;
        if (tid == 0 && a.state) {
            float *st4 = a.state + 4 * r;
            st4[0] = M; st4[1] = ST; st4[2] = S1; st4[3] = SO;
        }
    } else {
        const float *st4 = a.state + 4 * r;
        M = st4[0]; ST = st4[1]; S1 = st4[2]; SO = st4[3];
    }
    const bool none = padding || ST == 0.f;            // padding, or every logit masked: loss and gradient 0
    if (!(SO > 0.f)) rest = 0.0;

    if constexpr (MODE & DISTILL_LOSS) {
        const double log_st = log((double)ST);
        double term = 0.0;
        if (!none && p > 0.0) term = p * (log_p - (((double)row.load_one(place) - (double)M) / T - log_st));
        if (isnan(p)) term = p;
        double kl = block_sum<BLOCK>(term, dpart);
        if (tid == 0) {
            if (rest > 0.0) kl += rest * (log(rest) - log((double)SO) + log_st);
            double loss = 0.0;
            if (!none) {
                loss = (1.0 - (double)a.hard) * T * T * kl;
                if (a.hard == 1.f) loss = 0.0;
                if (hard_row) loss += (double)a.hard * (((double)M - (double)row.load_one(label)) + log((double)S1));
                if (isnan(ST)) loss = NAN;
            }
            a.loss[r] = (float)loss;
        }
    }

    // ---- backward ----
    if constexpr (MODE & DISTILL_GRAD) {
        const Row<DT> out(a.dlogits, r, a.dld, a.V);
        const double up = (double)a.scale * (a.dloss ? (double)a.dloss[r] : 1.0);
        const double soft = up * (1.0 - (double)a.hard) * T;
        const double cover = mass + rest;
        const float fq = none ? 0.f : (float)(soft * (cover - (rest > 0.0 ? rest * (double)ST / (double)SO : 0.0)) / (double)ST);
        const float f1 = none || !hard_row ? 0.f : (float)(up * (double)a.hard / (double)S1);
        auto put = [&](int j, float d) { out.base[out.shift + j] = Type::narrow(d); };
        for (int j = tid; j < a.V; j += BLOCK) {
            float d = 0.f;
            if (!none) {
                const float x = row.load_one(j) - M;
                d = fq * exp2_fast(x * c);
                if (hard_row) d = fmaf(f1, exp2_fast(x * c1), d);
            }
            put(j, d);
        }
        __syncthreads();                               // the places below are written again by other threads
        if (!none) {
            // the teacher's places and the label: each place once, by the first slot that names it
            auto fix = [&](int j, double target, bool is_label, bool top) {
                const double x = (double)row.load_one(j) - (double)M;
                double d = soft * ((top ? cover : cover - (rest > 0.0 ? rest * (double)ST / (double)SO : 0.0)) * exp(x / T) / (double)ST - target);
                if (hard_row) d += up * (double)a.hard * (exp(x) / (double)S1 - (is_label ? 1.0 : 0.0));
                put(j, (float)d);
            };
            if (place >= 0) {
                double target = 0.0;
                bool first = true;
                for (int i = 0; i < a.k; ++i) {
                    if (t.index[i] != place) continue;
                    if (i < tid) first = false;
                    target += t.p[i];
                }
                if (first) fix(place, target, hard_row && place == label, true);
            }
            if (hard_row && tid == 0) {
                bool taken = false;
                for (int i = 0; i < a.k; ++i) taken = taken || t.index[i] == label;
                if (!taken) fix(label, 0.0, true, false);
            }
        }
    }
}

struct DistillCall {
    const char *name;
    int dtype;
    size_t rows;
    DistillArgs a;
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
        !aligned_to(a.state, 4) || !aligned_to(a.dloss, 4))
        return fail(EASGD_EINVAL, "%s: indices, values, teacher_lse, labels, loss, state, dloss must be 4-byte aligned", q.name);
    if (mode & DISTILL_GRAD) {
        if (!std::isfinite(a.scale)) return fail(EASGD_EINVAL, "%s: scale must be finite", q.name);
        if (a.dld < (size_t)a.V) return fail(EASGD_EINVAL, "%s: dld (%zu) < V (%d)", q.name, a.dld, a.V);
        if (q.rows > 1 && a.dld > ((size_t)1 << 60) / q.rows) return fail(EASGD_ERANGE, "%s: rows * dld too large", q.name);
        if (!aligned_to(a.dlogits, dtype_bytes(q.dtype))) return fail(EASGD_EINVAL, "%s: dlogits must be aligned to its elements (%zu bytes)", q.name, dtype_bytes(q.dtype));
    }
    return EASGD_OK;
}

template <int MODE> static int launch_distill(const DistillCall &q, void *stream)
{
    if (int rc = check_distill(q, MODE)) return rc;
    clear_error();
    if (q.rows == 0) return EASGD_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(q.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const size_t bits = MODE & DISTILL_LOSS ? ((size_t)q.a.V + 16 + 31) / 32 * 4 : 0;
        if (q.a.teacher_lse) EASGD_LAUNCH((distill_rows_kernel<DT, 256, MODE, true>), dim3((unsigned)q.rows), dim3(256), bits, s, q.a);
        else EASGD_LAUNCH((distill_rows_kernel<DT, 256, MODE, false>), dim3((unsigned)q.rows), dim3(256), 0, s, q.a);
    });
    return check_launch(q.name);
}

}  // namespace easgd

extern "C" {

size_t easgd_distill_workspace_bytes(size_t, int, int) { return 0; }

int easgd_distill_loss(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                       const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, float *loss, float *state,
                       void *, size_t, void *stream)
{
    const easgd::DistillCall q = {"easgd_distill_loss", dtype, rows,
                                  {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, loss, state, nullptr, 1.f, nullptr, 0}};
    return easgd::launch_distill<easgd::DISTILL_LOSS>(q, stream);
}

int easgd_distill_grad(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                       const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, const float *state,
                       const float *dloss, float scale, void *dlogits, size_t dld, void *stream)
{
    const easgd::DistillCall q = {"easgd_distill_grad", dtype, rows,
                                  {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, nullptr,
                                   const_cast<float *>(state), dloss, scale, dlogits, dld}};
    return easgd::launch_distill<easgd::DISTILL_GRAD>(q, stream);
}

int easgd_distill(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *indices, const float *values,
                  const float *teacher_lse, int k, const int32_t *labels, float temperature, float hard, float scale, float *loss,
                  void *dlogits, size_t dld, void *, size_t, void *stream)
{
    const easgd::DistillCall q = {"easgd_distill", dtype, rows,
                                  {logits, ld, V, k, indices, values, teacher_lse, labels, temperature, hard, loss, nullptr, nullptr, scale, dlogits, dld}};
    return easgd::launch_distill<easgd::DISTILL_BOTH>(q, stream);
}

}  // extern "C"
