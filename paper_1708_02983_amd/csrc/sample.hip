// easgd_sample_tokens: one token of every row, drawn with a given random number.
#include "logits.h"
#include "logits_select.h"

namespace easgd {

struct SampleArgs {
    const void *logits;
    size_t ld;
    int V;
    const float *u, *temperature;
    const int *top_k;
    const float *top_p, *min_p;
    int *tokens;
    float *logprob;
    double unit;              // units of mass in the largest weight, a power of two
};

// w = exp((z - max) / T) as a whole number of units: adding 2^52 rounds to the nearest whole number and leaves it in the
// low bits of the sum (w * unit <= 2^51).
struct Weight {
    double inv_t, unit;
    float max;
    __device__ __forceinline__ double real(float z) const { return z == max ? 1.0 : exp(((double)z - (double)max) * inv_t); }
    __device__ __forceinline__ unsigned long long units(double w) const
    {
        return __builtin_bit_cast(unsigned long long, fma(w, unit, 0x1p52)) - 0x4330000000000000ull;
    }
    __device__ __forceinline__ unsigned long long operator()(float z) const { return units(real(z)); }
};

template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void sample_kernel(SampleArgs a)
{
    constexpr int VEC = Row<DT>::VEC, WAVES = BLOCK / 64;
    __shared__ SelectLds<true> sel;
    __shared__ unsigned long long part[WAVES];
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // the first token of the order
    unsigned long long first = 0;
    for (int s = tid; s < row.slots; s += BLOCK) {
        float x[VEC];
        Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const unsigned long long word = order_word(logit_key(x[i]), row.index(s, i));
            first = word > first ? word : first;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor(first, o);
        first = other > first ? other : first;
    }
    if (lane == 0) part[wave] = first;
    __syncthreads();
    for (int v = 0; v < WAVES; ++v) first = part[v] > first ? part[v] : first;
    __syncthreads();
    const float T = a.temperature ? a.temperature[r] : 1.f;
    if (first < FIRST_WORD || !(T > 0.f)) {
        if (tid == 0) {
            a.tokens[r] = first < FIRST_WORD ? -1 : (int)~(unsigned)first;
            if (a.logprob) a.logprob[r] = first < FIRST_WORD ? NAN : 0.f;
        }
        return;
    }
    const float max = key_logit((unsigned)(first >> 32));
    const Weight weight = {T == INFINITY && max == INFINITY ? 1.0 : 1.0 / (double)T, a.unit, max};      // a difference of -inf stays one
    unsigned long long floor = FIRST_WORD;
    const int top_k = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.f;
    const float min_p = a.min_p ? a.min_p[r] : 0.f;

    if (top_k >= 1 && top_k < a.V) {
        unsigned taken = 0;
        for (int s = tid; s < row.slots; s += BLOCK) {
            float x[VEC];
            Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) taken += logit_key(x[i]) != 0;
        }
        const unsigned long long n = block_sum<BLOCK>((unsigned long long)taken, part);
        if (n > (unsigned long long)top_k)
            floor = select_nth<BLOCK>(EachElement<DT, BLOCK>{row, 0, row.slots}, FIRST_WORD, top_k, sel);
    }
    if (top_p < 1.f) {
        unsigned long long mass = 0;
        for (int s = tid; s < row.slots; s += BLOCK) {
            float x[VEC];
            Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (order_word(logit_key(x[i]), row.index(s, i)) >= floor) mass += weight(x[i]);
        }
        mass = block_sum<BLOCK>(mass, part);
        const double target = ceil((double)top_p * (double)mass);
        floor = select_word<BLOCK, true>(EachElement<DT, BLOCK>{row, 0, row.slots}, floor, target >= 1.0 ? (unsigned long long)target : 1ull, sel, weight);
    }

    // the mass of what is kept, by wavefront: wavefront v owns a run of whole slots
    const int chunk = ((row.slots + BLOCK - 1) / BLOCK) * 64;
    const int s0 = wave * chunk, s1 = min(s0 + chunk, row.slots);
    auto kept_units = [&](float x, int index) -> unsigned long long {
        const unsigned long long word = order_word(logit_key(x), index);
        if (word < floor || word < FIRST_WORD) return 0;
        const double w = weight.real(x);
        return word == first || !(w < (double)min_p) ? weight.units(w) : 0;
    };
    auto slot_units = [&](int s) {
        unsigned long long u = 0;
        if (s < s1) {
            float x[VEC];
            Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) u += kept_units(x[i], row.index(s, i));
        }
        return u;
    };
    unsigned long long mass = 0;
    for (int s = s0 + lane; s < s1; s += 64) mass += slot_units(s);
    mass = wave_sum(mass);
    if (lane == 0) part[wave] = mass;
    __syncthreads();
    unsigned long long before = 0, total = 0;
    for (int v = 0; v < WAVES; ++v) {
        if (v < wave) before += part[v];
        total += part[v];
    }
    const float u = a.u[r];
    const double drawn = (double)(u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f) * (double)total;
    unsigned long long target = (unsigned long long)drawn;
    if (target >= total) target = total - 1;
    if (before > target || before + mass <= target) return;      // uniform for the wavefront: one is left
    for (int s = s0 + lane; s - lane < s1; s += 64) {
        const unsigned long long mine = slot_units(s);
        unsigned long long run = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned long long up = __shfl_up(run, o);
            if (lane >= o) run += up;
        }
        const unsigned long long all = __shfl(run, 63);
        if (before + all > target) {
            unsigned long long at = before + run - mine;
            if (at <= target && at + mine > target) {
                float x[VEC];
                Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const unsigned long long w = kept_units(x[i], row.index(s, i));
                    if (at <= target && at + w > target) {
                        a.tokens[r] = row.index(s, i);
                        if (a.logprob) a.logprob[r] = (float)log(weight.real(x[i]) * a.unit / (double)total);
                    }
                    at += w;
                }
            }
            return;
        }
        before += all;
    }
}

}  // namespace easgd

extern "C" {

size_t easgd_sample_tokens_workspace_bytes(size_t, int) { return 0; }

int easgd_sample_tokens(const void *logits, int dtype, size_t rows, int V, size_t ld, const float *u,
                        const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                        int32_t *tokens, float *logprob, void *, size_t, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_sample_tokens";
    if (int rc = check_logits(name, logits, dtype, rows, V, ld)) return rc;
    if (rows > 0 && (!u || !tokens)) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(u, 4) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) || !aligned_to(min_p, 4) ||
        !aligned_to(tokens, 4) || !aligned_to(logprob, 4))
        return fail(EASGD_EINVAL, "%s: u, temperature, top_k, top_p, min_p, tokens, logprob must be 4-byte aligned", name);
    clear_error();
    if (rows == 0) return EASGD_OK;
    int log2_v = 0;
    while ((1 << log2_v) < V) ++log2_v;
    const double unit = (double)(1ull << (62 - log2_v < 51 ? 62 - log2_v : 51));
    const SampleArgs a = {logits, ld, V, u, temperature, top_k, top_p, min_p, tokens, logprob, unit};
    by_dtype(dtype, [&](auto dt) {
        EASGD_LAUNCH((sample_kernel<decltype(dt)::value, 512>), dim3((unsigned)rows), dim3(512), 0, static_cast<hipStream_t>(stream), a);
    });
    return check_launch(name);
}

}  // extern "C"
