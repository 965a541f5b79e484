// easgd_top_logits: the k first logits of every row's order, and the row's log-sum-exp.
#include "logits.h"
#include "logits_select.h"

namespace easgd {

struct TopArgs {
    const void *logits;
    size_t ld;
    int V, k;
    float temperature;
    float *values;
    int *indices;
    float *lse;
};

template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void top_logits_kernel(TopArgs a)
{
    constexpr int VEC = Row<DT>::VEC;
    __shared__ SelectLds sel;
    __shared__ unsigned long long best[LOGITS_MAX_TOP];
    __shared__ float fpart[BLOCK / 64];
    __shared__ unsigned n_best;
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x;
    const float c = (float)(LOG2E / (double)a.temperature);

    float m = -FLT_MAX, sum = 0.f;
    unsigned taken = 0;
    for (int s = tid; s < row.slots; s += BLOCK) {
        float x[VEC];
        Row<DT>::Type::unpack(row.load(s), x);
        float top = x[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) top = fmaxf(top, x[i]);
        if (top > m) {
            sum *= exp2_fast((m - top) * c);
            m = top;
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            sum += exp2_fast((x[i] - m) * c);
            taken += logit_key(x[i]) != 0;
        }
    }
    const float M = block_max<BLOCK>(m, fpart);
    const float S = block_sum<BLOCK>(sum * exp2_fast((m - M) * c), fpart);
    const unsigned n = block_sum<BLOCK>(taken, reinterpret_cast<unsigned *>(fpart));
    if (a.lse && tid == 0) a.lse[r] = M == INFINITY ? INFINITY : (float)((double)M / (double)a.temperature + log((double)S));

    const unsigned want = n < (unsigned)a.k ? n : (unsigned)a.k;
    unsigned long long floor = FIRST_WORD;
    if (n > want) floor = select_word<DT, BLOCK, false>(row, FIRST_WORD, want, sel, [](float) { return 0ull; });
    if (tid == 0) n_best = 0;
    __syncthreads();
    for (int s = tid; s < row.slots; s += BLOCK) {
        float x[VEC];
        Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const unsigned long long word = order_word(logit_key(x[i]), row.index(s, i));
            if (word >= floor) {
                const unsigned at = atomicAdd(&n_best, 1u);
                if (at < LOGITS_MAX_TOP) best[at] = word;         // always, unless the logits change under the kernel
            }
        }
    }
    __syncthreads();
    // every word's rank is the number of larger ones
    for (int i = tid; i < a.k; i += BLOCK) {
        if (i < (int)want) {
            const unsigned long long mine = best[i];
            int rank = 0;
            for (unsigned j = 0; j < want; ++j) rank += best[j] > mine;
            a.values[r * a.k + rank] = key_logit((unsigned)(mine >> 32));
            a.indices[r * a.k + rank] = (int)~(unsigned)mine;
        } else {
            a.values[r * a.k + i] = -INFINITY;
            a.indices[r * a.k + i] = -1;
        }
    }
}

}  // namespace easgd

extern "C" {

size_t easgd_top_logits_workspace_bytes(size_t, int, int) { return 0; }

int easgd_top_logits(const void *logits, int dtype, size_t rows, int V, size_t ld, int k, float temperature,
                     float *values, int32_t *indices, float *lse, void *, size_t, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_top_logits";
    if (int rc = check_logits(name, logits, dtype, rows, V, ld)) return rc;
    if (k < 1 || k > LOGITS_MAX_TOP) return fail(EASGD_EINVAL, "%s: k must be in [1, %d], got %d", name, LOGITS_MAX_TOP, k);
    if (int rc = check_temperature(name, temperature)) return rc;
    if (rows > 0 && (!values || !indices)) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(values, 4) || !aligned_to(indices, 4) || !aligned_to(lse, 4)) return fail(EASGD_EINVAL, "%s: values, indices, lse must be 4-byte aligned", name);
    clear_error();
    if (rows == 0) return EASGD_OK;
    const TopArgs a = {logits, ld, V, k, temperature, values, indices, lse};
    by_dtype(dtype, [&](auto dt) {
        EASGD_LAUNCH((top_logits_kernel<decltype(dt)::value, 256>), dim3((unsigned)rows), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    });
    return check_launch(name);
}

}  // extern "C"
