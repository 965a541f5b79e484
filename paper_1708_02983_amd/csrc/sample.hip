// easgd_sample_tokens: one token of every row, drawn with a given random number.
//
// All three filters keep a prefix of the row's order, so what is kept is "every order word from some word on" (and w >= min_p),
// and the draw in index order needs no sorting: the kept mass by wavefront, then by 64 slots, then by element.  Masses are
// whole numbers of units, whose sums are the same in every order, so the passes over a row agree to the last bit.
//   top_k <= 256, or greedy:  the first k in one pass (logits_select.h), everything else on at most 256 words in LDS
//   top_p:                    the mass of the row in bins of equal width below the largest logit, then the bin of the border
//   neither:                  no border to find
// Bound: latency of the passes over a row (which stays in the caches) and, where masses of whole rows are asked for, the vector
// ALUs: some 25 instructions a logit for a 64-bit exponential.  A row is one block's, however few rows there are.  Measured (us a call,
// temperature 0.9, top_k 50 or 1000, top_p 0.9, min_p 0.05):
//   1 x 131072 bf16         none 35   top_k 27 / 74   top_p 97    min_p 18   greedy 12
//   256 x 131072 bf16       none 47   top_k 33 / 87   top_p 119   min_p 44   greedy 17
//   512 x 32000 fp16        none 27   top_k 21 / 44   top_p 55    min_p 21   greedy 11
//   2048 x 1000 fp32        none 15   top_k 24 / 15   top_p 28    min_p 16   greedy 13
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
    int unit;                 // log2 of the units of mass in the largest weight
};

// how many tokens the filters leave at most; 1 for greedy rows (and where nothing reaches a min_p above 1)
__device__ __forceinline__ int most_tokens(const SampleArgs &a, size_t r)
{
    const float T = a.temperature ? a.temperature[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    return T > 0.f && !(min_p > 1.f) ? (a.top_k ? a.top_k[r] : 0) : 1;
}

// w = 2^y with y = (z - max) log2(e) / T <= 0, in 64 bits: y = j / 512 + f with |f| <= 2^-10 (adding 1.5 * 2^43 rounds to the
// multiple of 2^-9 and leaves j in the low bits), 2^(j / 512) from a table in LDS and an exponent, 2^f from its Taylor polynomial,
// whose remainder is below (2^-10 ln 2)^4 / 24 = 9e-15.  (The time is the 64-bit instructions': 131072 logits on one compute unit
// 29 us; with 32 entries, as many copies as there are pairs of banks and polynomials of degree 5 33.)  Below 2^-200 the value no
// longer matters (a unit is at least 2^-51 of the largest weight, min_p at least 2^-149).
static constexpr int WEIGHT_TABLE = 512;
struct Weight {
    double scale, max;        // log2(e) / T
    float top;                // the largest logit
    int unit;
    bool infinite;            // the largest logit is +inf: logits are in or out
    const double *table;      // units of 2^(i / 512)
    __device__ __forceinline__ Weight(float T, float top, int unit, const double *table)
        : scale(LOG2E / (double)T), max((double)top), top(top), unit(unit), infinite(top == INFINITY), table(table) {}
    // every thread of the block; ends with a barrier
    template <int BLOCK> static __device__ __forceinline__ void fill(double *table, int unit)
    {
        for (int i = threadIdx.x; i < WEIGHT_TABLE; i += BLOCK) table[i] = power(unit) * exp2((double)i / WEIGHT_TABLE);
        __syncthreads();
    }
    static __device__ __forceinline__ double power(int n) { return __builtin_bit_cast(double, (unsigned long long)(n + 1023) << 52); }
    // 2^y units, not yet whole; no branch, so that the elements of a slot are computed side by side (256 rows of 131072 with
    // mixed filters: 109 us, 125 us with each element's own branches).  Product and sum stay two roundings wherever a logit's units are
    // asked for: joined in some places and not in others, two passes could disagree by a unit.
    __device__ __forceinline__ double scaled(float z) const
    {
#pragma clang fp contract(off)
        const double y = fmax(((double)z - max) * scale, -200.0), t = y + 0x1.8p43, f = y - (t - 0x1.8p43);
        const int j = (int)(unsigned)__builtin_bit_cast(unsigned long long, t);
        const unsigned long long e = __builtin_bit_cast(unsigned long long, table[j & (WEIGHT_TABLE - 1)]);
        const double a = __builtin_bit_cast(double, e + ((unsigned long long)(unsigned)((j >> 9) << 20) << 32));
        return a * fma(fma(fma(5.5504108664821576e-02, f, 2.4022650695910069e-01), f, 6.9314718055994529e-01), f, 1.0);
    }
    template <int VEC> __device__ __forceinline__ void scaled(const float (&z)[VEC], double (&w)[VEC]) const
    {
        if (infinite) {                                 // uniform: logits are in or out
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = z[i] == top ? power(unit) : 0.0;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = scaled(z[i]);
        }
    }
    // adding 2^52 rounds to the nearest whole number and leaves it in the low bits of the sum (units <= 2^51)
    static constexpr unsigned long long BIAS = 0x4330000000000000ull;
    static __device__ __forceinline__ unsigned long long biased(double w)
    {
#pragma clang fp contract(off)
        return __builtin_bit_cast(unsigned long long, w + 0x1p52);
    }
    __device__ __forceinline__ unsigned long long units(float z) const
    {
        const float one[1] = {z};
        double w[1];
        scaled<1>(one, w);
        return biased(w[0]) - BIAS;
    }
    __device__ __forceinline__ double real(float z) const
    {
        const float one[1] = {z};
        double w[1];
        scaled<1>(one, w);
        return w[0] * power(-unit);
    }
    // log of w over a mass
    __device__ __forceinline__ float log_share(float z, unsigned long long mass) const
    {
        const double ln_w = z == top ? 0.0 : ((double)z - max) * scale * 0.69314718055994530942;
        return (float)(ln_w - log((double)mass * power(-unit)));
    }
};

// exclusive sum over the threads of the block, and the sum of all; part: one word per wavefront.  Ends with a barrier.
template <int BLOCK>
__device__ __forceinline__ unsigned long long scan(unsigned long long v, unsigned long long *part, unsigned long long &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned long long run = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long up = __shfl_up(run, o);
        if (lane >= o) run += up;
    }
    if (lane == 63) part[wave] = run;
    __syncthreads();
    unsigned long long before = run - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < BLOCK / 64; ++w) {
        if (w < wave) before += part[w];
        all += part[w];
    }
    __syncthreads();
    return before;
}

// out[i], i < n: the number of j < n for which before(j, i) holds.  As many neighbouring lanes as there are threads share an i.
// Ends with a barrier.
template <int BLOCK, typename P> __device__ __forceinline__ void ranks(unsigned n, P before, unsigned *out)
{
    unsigned share = 1, log2_share = 0;
    while (share < 64 && 2 * share * n <= BLOCK) {
        share *= 2;
        ++log2_share;
    }
    for (unsigned t = threadIdx.x; t - (threadIdx.x & 63) < n * share; t += BLOCK) {       // whole wavefronts
        const unsigned i = t >> log2_share;
        unsigned rank = 0;
        if (i < n) {
#pragma unroll 4
            for (unsigned j = t & (share - 1); j < n; j += share) rank += before(j, i);
        }
        for (unsigned o = 1; o < share; o *= 2) rank += __shfl_xor(rank, o);
        if (i < n && (t & (share - 1)) == 0) out[i] = rank;
    }
    __syncthreads();
}

// the place of the drawn number in a mass: the token is the first at which the running sum exceeds it
__device__ __forceinline__ unsigned long long drawn(float u, unsigned long long mass)
{
    const double at = (double)(u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f) * (double)mass;
    const unsigned long long whole = (unsigned long long)at;
    return whole < mass ? whole : mass - 1;
}
// the mass that a prefix has to reach: top_p of `mass`, at least one unit
__device__ __forceinline__ unsigned long long wanted(float top_p, unsigned long long mass)
{
    const double target = ceil((double)top_p * (double)mass);
    return target >= 1.0 ? (unsigned long long)target : 1ull;
}

// Bins of equal width below the largest logit: 2047 of them over 18 units of T, the last for all that is further below.
static constexpr int MASS_BINS = SELECT_BINS, BORDER_LIST = TOP_LIST / 2;

union SampleLds {
    TopLds top;
    SelectLds<true> mass;
};

template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void sample_kernel(SampleArgs a)
{
    constexpr int VEC = Row<DT>::VEC, WAVES = BLOCK / 64;
    using Type = LogitType<DT>;
    __shared__ SampleLds lds;
    __shared__ unsigned long long part[WAVES];
    __shared__ unsigned long long mass_of[LOGITS_MAX_TOP];
    __shared__ float fpart[WAVES];
    __shared__ double table[WEIGHT_TABLE];
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float T = a.temperature ? a.temperature[r] : 1.f, top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];
    const int top_k = most_tokens(a, r);
    auto answer = [&](int token, float lp) {
        a.tokens[r] = token;
        if (a.logprob) a.logprob[r] = lp;
    };

    Weight::fill<BLOCK>(table, a.unit);

    // ---- few tokens: all further work is on their order words ----
    if (top_k >= 1 && top_k <= LOGITS_MAX_TOP) {
        const unsigned n = first_of<DT, BLOCK>(row, 0, row.slots, (unsigned)top_k, lds.top, [](const float (&)[VEC], int) {});
        if (n <= 1) {
            if (tid == 0) answer(n ? (int)~(unsigned)lds.top.list[0] : -1, n ? 0.f : NAN);
            return;
        }
        const unsigned i = tid;
        const unsigned long long *words = lds.top.list;
        const Weight weight(T, key_logit((unsigned)(words[0] >> 32)), a.unit, table);
        const float z = i < n ? key_logit((unsigned)(words[i] >> 32)) : 0.f;
        unsigned long long w = i < n ? weight.units(z) : 0, all;
        const unsigned long long before = scan<BLOCK>(w, part, all);
        bool keep = i < n;
        if (top_p < 1.f && before >= wanted(top_p, all)) keep = false;
        if (min_p > 0.f && i > 0 && i < n && weight.real(z) < (double)min_p) keep = false;
        if (!keep) w = 0;
        // by index
        unsigned *place = lds.top.select.count;
        ranks<BLOCK>(n, [&](unsigned j, unsigned q) { return (unsigned)words[j] > (unsigned)words[q]; }, place);      // words hold ~index
        const unsigned at = i < n ? place[i] : 0;
        if (i < n) mass_of[at] = w;
        __syncthreads();
        const unsigned long long w_at = i < n ? mass_of[i] : 0;
        const unsigned long long lead = scan<BLOCK>(w_at, part, all);
        if (i < n) mass_of[i] = lead;
        __syncthreads();
        const unsigned long long target = drawn(u, all);
        if (i < n && w && mass_of[at] <= target && target - mass_of[at] < w) answer((int)~(unsigned)words[i], weight.log_share(z, all));
        return;
    }

    // ---- the largest logit ----
    float M = -INFINITY;
    each_slot<DT, BLOCK>(row, 0, row.slots, [&](const uint4 &raw, int) {
        float x[VEC];
        Type::unpack(raw, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) M = fmaxf(M, x[i]);
    });
    M = block_max<BLOCK>(M, fpart);
    if (M == -INFINITY) {
        if (tid == 0) answer(-1, NAN);
        return;
    }
    const Weight weight(T, M, a.unit, table);
    unsigned long long floor = FIRST_WORD;

    // The word at which the weights (masses, or 1 each) of the words from `floor` on reach what `want` says of their sum (0: no
    // such border).  The weights are summed in bins of equal width below the largest logit; the bin of the border is listed, and
    // every listed word's sum of weights before it taken in the order.  Where the border is further below than the bins reach,
    // or its bin holds more words than the list, the order words are walked down digit by digit.
    auto border_word = [&](auto by_mass, float reach, auto want) -> unsigned long long {
        constexpr bool BY_MASS = decltype(by_mass)::value;
        auto weight_of = [&](float z) { return BY_MASS ? weight.units(z) : 1ull; };
        const float width = fminf((float)(MASS_BINS - 1) / reach, FLT_MAX);
        auto bin_of = [&](float z) {
            const float b = (M - z) * width;                        // descending logits have ascending bins, whatever is rounded
            return b < (float)(MASS_BINS - 1) ? (int)b : MASS_BINS - 1;      // NaN (+inf twice): the last
        };
        const float floor_logit = key_logit(max((unsigned)(floor >> 32), 0x00800000u));
        auto above_floor = [&](float z, int index) {                // the floor's index is the last of its value that counts
            return z > floor_logit || (z == floor_logit && (unsigned)index <= ~(unsigned)floor);
        };
        for (int b = tid; b < MASS_BINS; b += BLOCK) lds.mass.mass[b] = 0;
        __syncthreads();
        unsigned long long far = 0;
        each_slot<DT, BLOCK>(row, 0, row.slots, [&](const uint4 &raw, int s) {
            float x[VEC];
            double w[VEC];
            Type::unpack(raw, x);
            if constexpr (BY_MASS) weight.template scaled<VEC>(x, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                if (!above_floor(x[i], row.index(s, i))) continue;
                const unsigned long long weight_here = BY_MASS ? Weight::biased(w[i]) - Weight::BIAS : 1ull;
                const int b = bin_of(x[i]);
                if (b < MASS_BINS - 1) atomicAdd(&lds.mass.mass[b], weight_here);
                else far += weight_here;
            }
        });
        __syncthreads();
        constexpr int PER = MASS_BINS / BLOCK;
        unsigned long long w[PER], sum = 0, near;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            w[i] = lds.mass.mass[tid * PER + i];
            sum += w[i];
        }
        unsigned long long before = scan<BLOCK>(sum, part, near);
        const unsigned long long target = want(near + block_sum<BLOCK>(far, part));
        if (target == 0) return floor;
        if (tid == 0) lds.mass.bin = MASS_BINS - 1;
        __syncthreads();
        if (before < target && before + sum >= target) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < target && before + w[i] >= target) {
                    lds.mass.bin = (unsigned)(tid * PER + i);
                    lds.mass.above = before;
                }
                before += w[i];
            }
        }
        __syncthreads();
        const int border = (int)lds.mass.bin;
        const unsigned long long above = lds.mass.above;
        __syncthreads();
        if (border < MASS_BINS - 1) {
            if (tid == 0) {
                lds.top.n = 0;
                part[0] = floor;
            }
            __syncthreads();
            // logits of the border's bin, with room for the rounding of M - z and of its product
            const float middle = M - ((float)border + 0.5f) / width, half = (0.5f + (float)(border + 1) * 1e-6f) / width * 1.00001f + fabsf(M) * 1e-6f;
            each_slot<DT, BLOCK>(row, 0, row.slots, [&](const uint4 &raw, int s) {
                float x[VEC];
                Type::unpack(raw, x);
                bool any = false;
#pragma unroll
                for (int i = 0; i < VEC; ++i) any |= fabsf(x[i] - middle) <= half;
                if (!any) return;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    if (bin_of(x[i]) == border && above_floor(x[i], row.index(s, i))) {
                        const unsigned at = atomicAdd(&lds.top.n, 1u);
                        if (at < BORDER_LIST) lds.top.list[at] = order_word(logit_key(x[i]), row.index(s, i));
                    }
                }
            });
            __syncthreads();
            const unsigned n = lds.top.n;
            if (n <= BORDER_LIST) {
                unsigned long long *weights = lds.top.list + BORDER_LIST;
                for (unsigned i = tid; i < n; i += BLOCK) weights[i] = weight_of(key_logit((unsigned)(lds.top.list[i] >> 32)));
                __syncthreads();
                // as many neighbouring lanes to a word as there are threads
                unsigned share = 1;
                while (share < 64 && 2 * share * n <= BLOCK) share *= 2;
                for (unsigned t = tid; t - (t & 63) < n * share; t += BLOCK) {       // whole wavefronts
                    const unsigned i = t / share;
                    const unsigned long long mine = i < n ? lds.top.list[i] : 0;
                    unsigned long long lead = 0;
                    for (unsigned j = t % share; j < n; j += share) lead += lds.top.list[j] > mine ? weights[j] : 0;
                    for (unsigned o = 1; o < share; o *= 2) lead += __shfl_xor(lead, o);
                    lead += above;
                    if (i < n && t % share == 0 && lead < target && lead + weights[i] >= target) part[0] = mine;      // one word
                }
                __syncthreads();
                const unsigned long long found = part[0];
                __syncthreads();
                return found;
            }
        }
        __syncthreads();
        const EachElement<DT, BLOCK> elements{row, 0, row.slots};
        return select_word<BLOCK, BY_MASS>(elements, floor, target, lds.mass, weight_of);
    };
    const float cool = fminf(T, FLT_MAX / 32.f);
    if (top_k > LOGITS_MAX_TOP && top_k < a.V)
        floor = border_word(std::false_type{}, 18.f * fmaxf(cool, 1.f), [&](unsigned long long n) { return n > (unsigned long long)top_k ? (unsigned long long)top_k : 0ull; });
    if (top_p < 1.f)
        floor = border_word(std::true_type{}, 18.f * cool, [&](unsigned long long mass) { return wanted(top_p, mass); });

    // ---- the mass of what is kept, by wavefront: each owns a run of whole slots ----
    const int chunk = ((row.slots + BLOCK - 1) / BLOCK) * 64;
    const int s0 = wave * chunk, s1 = min(s0 + chunk, row.slots);
    // logits below `least` are not kept: the floor's, or what min_p leaves with room for rounding
    float least = key_logit(max((unsigned)(floor >> 32), 0x00800000u));
    if (min_p > 0.f && T < INFINITY) {
        const double edge = (double)M + (double)T * (log((double)fminf(min_p, 1.f)) * (1.0 + 1e-9) - 1e-9);
        least = fmaxf(least, (float)(edge - fabs(edge) * 1e-6));
    }
    const bool filtered = min_p > 0.f, whole = floor == FIRST_WORD && !filtered;
    const float floor_logit = key_logit(max((unsigned)(floor >> 32), 0x00800000u));
    const unsigned floor_index = ~(unsigned)floor;     // the last of the floor's value that is kept
    const double least_mass = (double)min_p * Weight::power(a.unit);
    // units of a slot's elements, 0 for those that are not kept
    auto kept_units = [&](const float (&x)[VEC], int s, unsigned long long (&u)[VEC]) {
        double w[VEC];
        weight.template scaled<VEC>(x, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const bool out = !(x[i] >= least) | ((x[i] == floor_logit) & ((unsigned)row.index(s, i) > floor_index)) |
                             (filtered & (w[i] < least_mass));
            u[i] = out ? 0 : Weight::biased(w[i]) - Weight::BIAS;
        }
    };
    auto slot_units = [&](const uint4 &raw, int s) {
        unsigned long long sum = 0;
        float x[VEC];
        Type::unpack(raw, x);
        if (whole) {                                    // uniform: masked logits (-inf and NaN) are all that is not kept
            double w[VEC];
            weight.template scaled<VEC>(x, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += x[i] >= -FLT_MAX ? Weight::biased(w[i]) : Weight::BIAS;
            return sum - VEC * Weight::BIAS;
        }
        float t = x[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) t = fmaxf(t, x[i]);
        if (t >= least) {
            unsigned long long u[VEC];
            kept_units(x, s, u);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += u[i];
        }
        return sum;
    };
    unsigned long long mass = 0;
    constexpr int DEEP = 8;
    for (int s = s0 + lane; s < s1; s += DEEP * 64) {
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if (s + i * 64 < s1) v[i] = row.load(s + i * 64);
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if (s + i * 64 < s1) mass += slot_units(v[i], s + i * 64);
    }
    mass = wave_sum(mass);
    if (lane == 0) part[wave] = mass;
    __syncthreads();
    unsigned long long before = 0, total = 0;
    for (int v = 0; v < WAVES; ++v) total += part[v];
    const unsigned long long target = drawn(u, total);
    int chosen = 0;
    while (chosen < WAVES - 1 && before + part[chosen] <= target) before += part[chosen++];
    __syncthreads();
    // the chosen wavefront's run, a slot per thread of the whole block
    const int end = min((chosen + 1) * chunk, row.slots);
    for (int s = chosen * chunk + tid; s - tid < end; s += BLOCK) {            // uniform
        uint4 raw = Row<DT>::empty();
        unsigned long long mine = 0, all;
        if (s < end) {
            raw = row.load(s);
            mine = slot_units(raw, s);
        }
        unsigned long long at = before + scan<BLOCK>(mine, part, all);
        if (at <= target && target - at < mine) {
            float x[VEC];
            unsigned long long w[VEC];
            Type::unpack(raw, x);
            kept_units(x, s, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                if (at <= target && target - at < w[i]) answer(row.index(s, i), weight.log_share(x[i], total));
                at += w[i];
            }
        }
        before += all;
        if (before > target) return;
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
    const SampleArgs a = {logits, ld, V, u, temperature, top_k, top_p, min_p, tokens, logprob, 62 - log2_v < 51 ? 62 - log2_v : 51};
    const int slots = most_slots(dtype, V);
    by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto launch = [&](auto block) {
            constexpr int BLOCK = decltype(block)::value;
            EASGD_LAUNCH((sample_kernel<DT, BLOCK>), dim3((unsigned)rows), dim3(BLOCK), 0, static_cast<hipStream_t>(stream), a);
        };
        if (slots <= 1024) launch(std::integral_constant<int, 256>{});
        else if (slots <= 4096) launch(std::integral_constant<int, 512>{});
        else launch(std::integral_constant<int, 1024>{});
    });
    return check_launch(name);
}

}  // extern "C"
