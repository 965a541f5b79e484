// Tokens that are given: their log probabilities, the rows' entropies, ranks and first alternatives, and the gradients of all that.
//
// Per row (see include/easgd.h for the definition): with a reference m near the largest logit, y_j = (z_j - m) log2(e) / T and
// e_j = 2^y_j,
//   s = sum e_j, u = sum e_j y_j:  logprob = (z_t - m)/T - ln s,  entropy H = ln s - ln2 u / s  (the same for any m),
//   d/dz_j of gl logprob + gh H  =  e_j (A + B y_j) + [j = t] gl / T  with  A = (-gl - gh (H - ln s)) / (s T), B = -gh ln2 / (s T),
// so sums and gradients are one pass each, with one exponential and a few fused multiply-adds a logit.  Bound: HBM for many long rows
// (each logit once in, each gradient once out), latency for few or short ones.
#include "score.h"
#include "logits_grad.h"
#include "logits_select.h"
#include "row_sums.h"

namespace easgd {

struct ScoreArgs {
    const void *logits;
    size_t ld, rows;
    int V;
    const int *tokens;
    float temperature;
    float *logprob, *entropy;
    int *rank;
    int k;
    float *top_logprob;
    int *top_indices;
    float4 *state;
    const float *weight;           // easgd_token_loss: the loss is -weight logprob - bonus H
    float bonus;
    float *loss;
    const float *dlogprob, *dentropy;
    float scale;
    void *dlogits;
    size_t dld;
    int parts;                     // logits are the sum of this many matrices (fp32, short rows)
    size_t part_stride;
    int segments, seg_slots;       // slots of a part of a row
    float4 *partial;               // [rows][segments]: (m, s, u, logits before the token) of a part of a row
    unsigned long long *words;     // [rows][segments][k]: the first k of every part (0: none left)
};

static constexpr float LN2 = 0.693147180559945309f;
static constexpr double LN2_64 = 0.69314718055994530942;
// the exponent that stands for any smaller one in e_j y_j, where e_j is 0: a masked place must not make it 0 times infinity
static constexpr float LEAST = -256.f;

// The hardware's product in which 0 times anything, infinities and NaN among it, is 0.
extern "C" __device__ float mul_zero_first(float, float) __asm("llvm.amdgcn.fmul.legacy");

// ---- sums ----------------------------------------------------------------------------------------------------------------
// Running sums of a thread relative to a reference that its wavefront shares (Reference in row_sums.h): the largest logit of the
// first slots that hold any, moved when a slot's exponentials sum up to more than 2^12, so that the usual slot needs neither a
// maximum nor a rescaling.  u is then off by at most 12 units of rounding of s, which the entropy divides by s.
template <int VEC, bool ENTROPY> struct TokenSums {
    const Scales &q;
    Reference<VEC> at;
    float s = 0.f, u = 0.f;

    __device__ __forceinline__ explicit TokenSums(const Scales &q) : q(q), at(q) {}
    // whole wavefronts call it (lanes without a slot with an empty one); returns the slot's sum
    __device__ __forceinline__ float add(const float (&x)[VEC])
    {
        float sum = 0.f, more = 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float y = fmaf(x[i], at.c, -at.rc), e = exp2_fast(y);
            sum += e;
            if constexpr (ENTROPY) more = fmaf(e, y, more);
        }
        // NaN in either: a masked place, among others
        const bool fine = at.ref > -INFINITY && sum <= 0x1p12f && (!ENTROPY || more <= 0x1p30f);
        if (__any(!fine)) careful(x, sum, more);        // uniform for the wavefront
        s += sum;
        if constexpr (ENTROPY) u += more;
        return sum;
    }
    // below it, the sum of a slot has no exponential of a logit from z on (exponentials are right to a few units)
    __device__ __forceinline__ float bar(float z) const { return exp2_fast(fmaf(z, at.c, -at.rc)) * (1.f - 0x1p-16f); }
    // a slot whose sums are not as they should be: the first one, a logit far above the reference, masked places, NaN, large logits
    __device__ __forceinline__ void careful(const float (&x)[VEC], float &sum, float &more)
    {
        float t = x[0];
        bool odd = isnan(x[0]);
#pragma unroll
        for (int i = 1; i < VEC; ++i) {
            t = fmaxf(t, x[i]);
            odd = odd || isnan(x[i]);
        }
        t = uniform(wave_max(t));
        if (t > at.ref && (at.ref == -INFINITY || __any(!(sum <= 0x1p12f)))) {
            const Reference<VEC> old = at;
            at.set(t, q);
            if (old.ref > -INFINITY) {                  // what the exponents of before are now
                const float up = fmaxf((old.ref - at.ref) * q.c - old.lost + at.lost, -1e4f), f = exp2_fast(up);
                if constexpr (ENTROPY) u = f * fmaf(up, s, u);
                s *= f;
            }
        }
        sum = odd ? NAN : 0.f;
        more = 0.f;
        if (at.ref == -INFINITY) return;                // masked places only, so far
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float y = at.by_difference() ? (x[i] - at.ref) * q.c : fmaf(x[i], at.c, -at.rc), e = exp2_fast(y);
            sum += e;
            if constexpr (ENTROPY) more = fmaf(e, fmaxf(y, LEAST), more);
        }
    }
    // sums (m, s, u, 0) of a wavefront, without what rounding rc added to the exponents
    __device__ __forceinline__ float4 of_wave() const
    {
        const float f = exp2_fast(-at.lost), ws = wave_sum(s), wu = ENTROPY ? wave_sum(u) : 0.f;
        return make_float4(at.ref, ws * f, ENTROPY ? f * fmaf(-at.lost, ws, wu) : 0.f, 0.f);
    }
};

// a part's sums, relative to its own reference, as they are relative to m, which is at least as large
__device__ __forceinline__ float4 rebased(const float4 &p, float m, const Scales &q)
{
    const float up = p.x == m || p.x == -INFINITY ? 0.f : fmaxf((p.x - m) * q.c, -1e4f), f = exp2_fast(up);
    return make_float4(m, p.y * f, f * fmaf(up, p.y, p.z), p.w);
}

// ---- ranks -----------------------------------------------------------------------------------------------------------------
// How many logits of the row come before the token in its order: z > z_t, or z == z_t at a lower index.  Slots before the
// token's compare with z >= z_t, slots behind it with z >= the next larger number, and the token's own slot looks closely.
// A slot whose sum of exponentials is below the token's own has nothing to count: one comparison a slot for tokens of any standing.
struct RankCount {
    float z, from;             // of the token; the next larger number
    float ref = NAN, bar = 0.f;      // the reference of the sums for which `bar` is the token's
    int slot, index;           // of the token
    unsigned n = 0;            // of this lane
    template <int DT> __device__ __forceinline__ void set(const Row<DT> &row, int token)
    {
        slot = (token + row.shift) / Row<DT>::VEC;
        index = token;
        z = row.load_one(token);
        if (!(z > -INFINITY)) z = from = -FLT_MAX;      // a masked token: behind all that are not
        else if (z == INFINITY) from = NAN;
        else {
            const unsigned b = __float_as_uint(z + 0.f);
            from = z == 0.f ? __uint_as_float(1u) : __uint_as_float(b & 0x80000000u ? b - 1 : b + 1);
        }
    }
    template <int DT, typename S> __device__ __forceinline__ void add(const Row<DT> &row, const float (&x)[Row<DT>::VEC], int s, float sum, const S &sums)
    {
        if (sums.at.ref != ref) {                       // uniform, and rare
            ref = sums.at.ref;
            bar = sums.bar(z);
        }
        if (!__any(!(sum < bar))) return;               // uniform for the wavefront
        const float least = s < slot ? z : from;
        if (__any(s == slot)) {
#pragma unroll
            for (int i = 0; i < Row<DT>::VEC; ++i) n += x[i] >= (s == slot && row.index(s, i) < index ? z : least);
        } else {
#pragma unroll
            for (int i = 0; i < Row<DT>::VEC; ++i) n += x[i] >= least;
        }
    }
};

// ---- results of a row ------------------------------------------------------------------------------------------------------
// What the sums of a row say: ln s and the entropy.
struct RowScore {
    double log_s, entropy;
    bool none;                 // every logit masked
    __device__ __forceinline__ explicit RowScore(const float4 &w)
    {
        none = w.y == 0.f;
        log_s = none ? 0.0 : log((double)w.y);
        const double h = log_s - LN2_64 * (double)w.z / (double)w.y;
        entropy = none || h < 0.0 ? 0.0 : h;
    }
};
__device__ __forceinline__ double log_probability(const RowScore &row, float m, float z, float temperature)
{
    return row.none ? -(double)INFINITY : ((double)z - (double)m) / (double)temperature - row.log_s;
}
// One thread.  token: whether the row has one.
__device__ __forceinline__ void write_score(const ScoreArgs &a, size_t r, bool padding, bool token, const float4 &w, float z_token, unsigned before)
{
    const RowScore row(w);
    const double lp = token ? log_probability(row, w.x, z_token, a.temperature) : 0.0;
    if (a.logprob) a.logprob[r] = padding ? 0.f : (float)lp;
    if (a.entropy) a.entropy[r] = padding ? 0.f : (float)row.entropy;
    if (a.rank) a.rank[r] = padding ? -1 : (int)before;
    if (a.state) a.state[r] = padding ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(w.x, w.y, (float)row.entropy, 0.f);
    if (a.loss) {
        const float weight = a.weight ? a.weight[r] : 1.f;
        double loss = weight != 0.f ? -(double)weight * lp : 0.0;
        if (a.bonus != 0.f) loss -= (double)a.bonus * row.entropy;
        if (isnan(w.y)) loss = NAN;
        a.loss[r] = padding || row.none ? 0.f : (float)loss;
    }
}
// an alternative from its order word (0: none left)
__device__ __forceinline__ void write_alternative(const ScoreArgs &a, size_t r, unsigned at, unsigned long long word, const RowScore &row, float m)
{
    a.top_logprob[r * a.k + at] = word ? (float)log_probability(row, m, key_logit((unsigned)(word >> 32)), a.temperature) : -INFINITY;
    a.top_indices[r * a.k + at] = word ? (int)~(unsigned)word : -1;
}
__device__ __forceinline__ bool padded(const ScoreArgs &a, int token) { return a.tokens && (unsigned)token >= (unsigned)a.V; }
template <int BLOCK> __device__ __forceinline__ void write_padding(const ScoreArgs &a, size_t r)
{
    if (threadIdx.x == 0) write_score(a, r, true, false, make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0);
    for (int i = threadIdx.x; i < a.k; i += BLOCK) write_alternative(a, r, i, 0, RowScore(make_float4(0.f, 0.f, 0.f, 0.f)), 0.f);
}

// ---- sums of rows, or of parts of rows, a block each --------------------------------------------------------------------------
// Every slot of [s0, s1) through whole wavefronts, DEEP loads ahead: f(raw, slot), an empty slot where a lane has none.
template <int DT, int BLOCK, int DEEP, bool ONCE, typename F> __device__ __forceinline__ void walk(const Row<DT> &row, int s0, int s1, F f)
{
    uint4 v[DEEP];
    int s = s0 + (int)threadIdx.x;
    const int lead = s0 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x & ~63);
    auto load = [&](int s, int first) {                 // first: of the wavefront
        if (first * Row<DT>::VEC >= row.shift && first + 64 <= s1 && (first + 64) * Row<DT>::VEC <= row.end) return ONCE ? row.load_once(s) : row.load_full(s);
        return s < s1 ? row.load(s) : row.empty();
    };
#pragma unroll
    for (int i = 0; i < DEEP; ++i) v[i] = load(s + i * BLOCK, lead + i * BLOCK);
    for (int first = lead; first < s1; first += DEEP * BLOCK, s += DEEP * BLOCK) {
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            if (first + i * BLOCK >= s1) break;         // uniform: the whole wavefront is behind the end
            f(v[i], s + i * BLOCK);
            if (first + (DEEP + i) * BLOCK < s1) v[i] = load(s + (DEEP + i) * BLOCK, first + (DEEP + i) * BLOCK);
        }
    }
}

template <int BLOCK> struct JoinLds {
    float4 part[BLOCK / 64];
};
// the sums of a block's wavefronts (w: of this one; the last number counts), for every thread
template <int BLOCK> __device__ __forceinline__ float4 join_waves(float4 w, JoinLds<BLOCK> &lds, const Scales &q)
{
    constexpr int WAVES = BLOCK / 64;
    __syncthreads();                                    // everyone is done with the sums before these
    if ((threadIdx.x & 63) == 0) lds.part[threadIdx.x >> 6] = w;
    __syncthreads();
    w = lds.part[threadIdx.x & (WAVES - 1)];
    unsigned n = __float_as_uint(w.w);
    float m = w.x;
#pragma unroll
    for (int o = WAVES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    w = rebased(w, m, q);
#pragma unroll
    for (int o = WAVES / 2; o > 0; o >>= 1) {
        w.y += __shfl_xor(w.y, o);
        w.z += __shfl_xor(w.z, o);
        n += __shfl_xor(n, o);
    }
    w.w = __uint_as_float(n);
    return w;
}
template <int BLOCK, typename S> __device__ __forceinline__ float4 block_sums(const S &sums, unsigned before, JoinLds<BLOCK> &lds, const Scales &q)
{
    float4 w = sums.of_wave();
    w.w = __uint_as_float(before);
    return join_waves<BLOCK>(w, lds, q);
}

// Bound: HBM, the vector ALUs 70 % busy with ranks.  2048 x 131072 bf16, call after call: 87 us = 6.2 TB/s, with ranks 104 (blocks of 512 or 1024 threads the same; loads
// that stay in the caches 98).
template <int DT, int BLOCK, bool ENTROPY, bool RANK, bool ONCE>
__global__ __launch_bounds__(BLOCK) void score_rows_kernel(ScoreArgs a)
{
    constexpr int VEC = Row<DT>::VEC;
    __shared__ JoinLds<BLOCK> lds;
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int token = a.tokens ? a.tokens[r] : 0;
    if (padded(a, token)) {
        if (a.segments == 1) write_padding<BLOCK>(a, r);
        return;
    }
    const Scales q(a.temperature);
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    TokenSums<VEC, ENTROPY> sums(q);
    RankCount rank;
    if constexpr (RANK) rank.set(row, token);
    walk<DT, BLOCK, 4, ONCE>(row, s0, s1, [&](const uint4 &raw, int s) {
        float x[VEC];
        Row<DT>::Type::unpack(raw, x);
        const float sum = sums.add(x);
        if constexpr (RANK) rank.add(row, x, s, sum, sums);
    });
    const float4 w = block_sums<BLOCK>(sums, RANK ? wave_sum(rank.n) : 0u, lds, q);
    if (threadIdx.x != 0) return;
    if (a.segments > 1) a.partial[blockIdx.x] = w;
    else write_score(a, r, false, a.tokens, w, a.tokens ? row.load_one(token) : 0.f, __float_as_uint(w.w));
}

// The same with the first k.  Bound: latency for few rows (48 x 50001 fp16, k = 20: 13.3 us, and 4.7 for the join), selection for many (first_of).
template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void score_top_kernel(ScoreArgs a)
{
    constexpr int VEC = Row<DT>::VEC;
    __shared__ TopLds top;
    __shared__ JoinLds<BLOCK> lds;
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int token = a.tokens ? a.tokens[r] : 0;
    if (padded(a, token)) {
        if (a.segments == 1) write_padding<BLOCK>(a, r);
        return;
    }
    const Scales q(a.temperature);
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    TokenSums<VEC, true> sums(q);
    RankCount rank;
    rank.set(row, token);
    const unsigned n = first_of<DT, BLOCK>(row, s0, s1, (unsigned)a.k, top, [&](const float (&x)[VEC], int s) {
        rank.add(row, x, s, sums.add(x), sums);
    });
    const float4 w = block_sums<BLOCK>(sums, wave_sum(rank.n), lds, q);
    const unsigned i = threadIdx.x;
    if (a.segments > 1) {
        if (i == 0) a.partial[blockIdx.x] = w;
        if (i < (unsigned)a.k) a.words[(size_t)blockIdx.x * a.k + i] = i < n ? top.list[i] : 0;
        return;
    }
    if (i == 0) write_score(a, r, false, a.tokens, w, a.tokens ? row.load_one(token) : 0.f, __float_as_uint(w.w));
    if (i < (unsigned)a.k) write_alternative(a, r, i, i < n ? top.list[i] : 0, RowScore(w), w.x);
}

// ---- the parts of a row together ------------------------------------------------------------------------------------------------
// the sums of a row's parts, a part per lane (and every 64th after it), in a fixed order, for every lane of a wavefront
__device__ __forceinline__ float4 join_parts(const ScoreArgs &a, size_t r, const Scales &q)
{
    const int lane = threadIdx.x & 63;
    const float4 *parts = a.partial + r * a.segments;
    float4 own = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    unsigned before = 0;
    for (int i = lane; i < a.segments; i += 64) {
        const float4 p = parts[i], w = own;
        const float m = fmaxf(w.x, p.x);
        const float4 x = rebased(w, m, q), y = rebased(p, m, q);
        own = make_float4(m, x.y + y.y, x.z + y.z, 0.f);
        before += __float_as_uint(p.w);
    }
    const float m = wave_max(own.x);
    own = rebased(own, m, q);
    return make_float4(m, wave_sum(own.y), wave_sum(own.z), __uint_as_float(wave_sum(before)));
}

template <int DT>
__global__ __launch_bounds__(64) void score_join_kernel(ScoreArgs a)
{
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int token = a.tokens ? a.tokens[r] : 0;
    if (padded(a, token)) {
        write_padding<64>(a, r);
        return;
    }
    const float z_token = a.tokens ? row.load_one(token) : 0.f;
    const float4 w = join_parts(a, r, Scales(a.temperature));
    if (threadIdx.x == 0) write_score(a, r, false, a.tokens, w, z_token, __float_as_uint(w.w));
}

template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void score_top_join_kernel(ScoreArgs a)
{
    __shared__ TopLds top;
    __shared__ float4 sums;
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int token = a.tokens ? a.tokens[r] : 0;
    if (padded(a, token)) {
        write_padding<BLOCK>(a, r);
        return;
    }
    const unsigned all = (unsigned)(a.segments * a.k);             // <= TOP_LIST
    if (threadIdx.x < 64) {
        const float4 w = join_parts(a, r, Scales(a.temperature));
        if (threadIdx.x == 0) {
            sums = w;
            write_score(a, r, false, a.tokens, w, a.tokens ? row.load_one(token) : 0.f, __float_as_uint(w.w));
        }
    }
    if (threadIdx.x == 0) top.n = all;
    for (unsigned i = threadIdx.x; i < all; i += BLOCK) top.list[i] = a.words[r * all + i];
    __syncthreads();
    if (all <= BLOCK) {                                 // a look at every pair: places that are left over are 0, behind all words
        const unsigned long long word = threadIdx.x < all ? top.list[threadIdx.x] : 0;
        unsigned at = 0, there = 0;
#pragma unroll 8
        for (unsigned i = 0; i < all; ++i) {
            const unsigned long long other = top.list[i];
            at += other > word;
            there += other != 0;
        }
        const RowScore score(sums);
        if (word && at < (unsigned)a.k) write_alternative(a, r, at, word, score, sums.x);
        if (threadIdx.x >= there && threadIdx.x < (unsigned)a.k) write_alternative(a, r, threadIdx.x, 0, score, sums.x);
        return;
    }
    unsigned n = keep_from<BLOCK>(top, all, FIRST_WORD);           // the words that are there
    if (n > 512) n = keep_from<BLOCK>(top, n, select_nth<BLOCK>(EachListed{top.list, n, BLOCK}, FIRST_WORD, a.k, top.select));
    rank_list<BLOCK>(top, n, a.k);
    const unsigned i = threadIdx.x;
    if (i < (unsigned)a.k) write_alternative(a, r, i, i < n ? top.list[i] : 0, RowScore(sums), sums.x);
}

// ---- gradients -----------------------------------------------------------------------------------------------------------------
// The gradient of a row from its reference, sum and mean exponent (u / s), as a function of the logit.  log q[j] + H is ln2 (y_j - u / s):
// no logarithm is taken, and nothing here needs 64 bits.
template <int VEC> struct TokenSlope {
    Reference<VEC> at;
    float a, b, of_token;
    bool none;                 // nothing to learn: the gradient is 0
    // differences: of() is not called; exponents are those of exact differences to m
    __device__ __forceinline__ TokenSlope(const ScoreArgs &args, size_t r, bool padding, float m, float sum, float mean, float z_token, const Scales &q,
                                          bool differences = false)
        : at(uniform(m), q)
    {
        none = padding || sum == 0.f;
        float gl, gh;
        if (args.loss) {
            gl = -args.scale * (args.weight ? args.weight[r] : 1.f);
            gh = -args.scale * args.bonus * LN2;
        } else {
            gl = args.dlogprob ? args.scale * args.dlogprob[r] : 0.f;
            gh = args.dentropy ? args.scale * args.dentropy[r] * LN2 : 0.f;
        }
        const float by_T = 1.f / args.temperature, by_sum = 1.f / sum;
        const float lost = differences ? 0.f : at.lost, factor = by_T * by_sum * (differences ? 1.f : exp2_fast(-at.lost));
        a = uniform(fmaf(gh, mean + lost, -gl) * factor);
        b = uniform(-gh * factor);
        const float y = (z_token - m) * q.c, p = exp2_fast(y) * by_sum;
        of_token = uniform((gl * (1.f - p) - (p > 0.f ? gh * p * (y - mean) : 0.f)) * by_T);
        if (isnan(sum)) {                               // a row with a NaN or +inf: every exponential is 1, or NaN, and a and b are NaN
            of_token = NAN;
            at.c = at.rc = 0.f;
        }
    }
    // A masked place has e = 0 and y = -inf: the product in which 0 times anything is 0.
    template <bool ENTROPY> __device__ __forceinline__ void of(float (&x)[VEC]) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float y = fmaf(x[i], at.c, -at.rc), e = exp2_fast(y);
            x[i] = ENTROPY ? mul_zero_first(e, fmaf(b, y, a)) : e * a;
        }
    }
    // where the reference asks for it (large logits)
    __device__ __forceinline__ void of_difference(float (&x)[VEC], const Scales &q) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float y = (x[i] - at.ref) * q.c;
            x[i] = mul_zero_first(exp2_fast(y), fmaf(b, y, a));
        }
    }
};

// The token's own gradient among those of a slot.
template <int DT> struct TokenPlace {
    static constexpr int VEC = Row<DT>::VEC;
    const Row<DT> &row;
    int token, slot;           // slot -1: the row has no token
    float d;
    __device__ __forceinline__ TokenPlace(const Row<DT> &row, int token, float d)
        : row(row), token(token), slot(token < 0 ? -1 : (int)((unsigned)(token + row.shift) / VEC)), d(d) {}
    __device__ __forceinline__ void put(float (&x)[VEC], int s) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = s == slot && row.index(s, i) == token ? d : x[i];
    }
};

// u / s from the sum and the entropy that the forward pass left
__device__ __forceinline__ float mean_exponent(float sum, float entropy) { return (float)((log((double)sum) - (double)entropy) / LN2_64); }

// full slot `from` + thread, read once: a uniform address and an offset
template <int DT> __device__ __forceinline__ uint4 load_at(const Row<DT> &row, int from)
{
    typedef unsigned Words __attribute__((ext_vector_type(4)));
    const Words w = __builtin_nontemporal_load(reinterpret_cast<const Words *>(row.base) + from + (unsigned)threadIdx.x);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One pass, each part of a row by a block.  Bound: HBM.  1024 x 32000 bf16 with entropies 22 us = 5.9 TB/s, 777 x 50001 fp16 without 25 us = 6.1 TB/s,
// 2048 x 131072 bf16 with entropies 196 us = 5.5 TB/s.
template <int DT, int BLOCK, bool ENTROPY, bool ONCE>
__global__ __launch_bounds__(BLOCK, 8) void score_grad_kernel(ScoreArgs a)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const int token = a.tokens ? a.tokens[r] : -1;
    const bool padding = padded(a, token);
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    const GradRow<DT> out(a.dlogits, a.dld, a.V, r, row);
    if (padding) {
        out.clear(s1, BLOCK, s0);
        return;
    }
    const Scales q(a.temperature);
    const float4 state = a.state[r];
    const TokenSlope<VEC> g(a, r, padding, state.x, state.y, mean_exponent(state.y, state.z), a.tokens ? row.load_one(token) : 0.f, q);
    if (g.none) {
        out.clear(s1, BLOCK, s0);
        return;
    }
    const TokenPlace<DT> place(row, token, g.of_token);
    auto careful = [&](int s) {                         // any slot, in any way
        float x[VEC];
        Row<DT>::Type::unpack(row.load(s), x);
        if (g.at.by_difference()) g.of_difference(x, q);
        else g.template of<ENTROPY>(x);
        place.put(x, s);
        out.store(s, x, row.full(s));
    };
    if (g.at.by_difference() || !out.same) {            // uniform, and rare
#pragma unroll 1
        for (int s = s0 + (int)threadIdx.x; s < s1; s += BLOCK) careful(s);
        return;
    }
    const int f0 = max(s0, row.first_full()), f1 = min(s1, row.end_full()), wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x & ~63u);
    if (threadIdx.x == 0 && s0 == 0 && s1 > 0 && row.shift) careful(0);
    if (threadIdx.x == 1 && s0 < s1 && s1 == row.slots && row.slots > row.end_full() && (row.slots > 1 || !row.shift)) careful(row.slots - 1);
    auto put = [&](const uint4 &raw, int from) {        // full slot `from` + thread
        float x[VEC];
        Row<DT>::Type::unpack(raw, x);
        g.template of<ENTROPY>(x);
        if ((unsigned)(place.slot - (from + wave)) < 64u) place.put(x, from + (int)threadIdx.x);         // uniform for the wavefront
        out.store_at(from, x);
    };
    int from = f0;
    for (; from + DEEP * BLOCK <= f1; from += DEEP * BLOCK) {
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) v[i] = ONCE ? load_at(row, from + i * BLOCK) : row.load_full(from + i * BLOCK + (int)threadIdx.x);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) put(v[i], from + i * BLOCK);
    }
    uint4 v[DEEP];
#pragma unroll
    for (int i = 0; i < DEEP; ++i)
        if (from + i * BLOCK + (int)threadIdx.x < f1) v[i] = ONCE ? load_at(row, from + i * BLOCK) : row.load_full(from + i * BLOCK + (int)threadIdx.x);
#pragma unroll
    for (int i = 0; i < DEEP; ++i)
        if (from + i * BLOCK + (int)threadIdx.x < f1) put(v[i], from + i * BLOCK);
}

// ---- loss and gradient in one pass over memory -----------------------------------------------------------------------------------
// A block holds its row between the sums and the gradient, NV slots a thread in registers and NL in LDS; what is longer is read again, from the
// caches.  Bound: the vector ALUs (an exponential takes four issue slots and either pass has one: 16 slots a logit with an entropy) and HBM in turn, since
// all of a block waits for its sums.  2048 x 131072 bf16 with entropies 204 us = 5.3 TB/s call after call on the same logits, 228 on logits that were written just
// before (sums and gradients as two launches 287), without entropies 181; 1024 x 65536 fp32, half the bytes and a quarter of the exponentials, 93 us = 5.8 TB/s;
// 777 x 50001 fp16 34 us; 4096 x 2000 bf16 16 to 20 us.
//
// The sums of a wavefront's slots relative to the largest logit of its first slots, without a look at each; where they come out wrong (a lane's sum above
// 2^12, as by a logit 8.3 T above that one; large logits, NaN; with entropies masked places, 0 times infinity), once more relative to the largest of all,
// which takes two further passes over the wavefront's slots.  With entropies an empty slot of a lane is a masked place, too: the first wavefront of every
// row, whose lanes without a partial slot at the row's ends hold an empty one, and a wavefront whose last slots are not all there always take them, while the others
// wait for their sums.
template <int DT, int BLOCK, int NV, int NL, bool ENTROPY> struct HeldRow {
    using Type = LogitType<DT>;
    static constexpr int VEC = Type::VEC;
    uint4 v[NV], edge;
    uint4 *own;                // in LDS: slot NV + k of this thread at own[k * BLOCK]
    // full slots [f0, f1): thread t has f0 + t + i * BLOCK; threads 0 and 1 have the partial slots at the row's ends
    __device__ __forceinline__ void fetch(const Row<DT> &row, int i)
    {
        const int from = row.first_full() + i * BLOCK;
        if (lead(row) + i * BLOCK < row.end_full()) v[i] = from + (int)threadIdx.x < row.end_full() ? load_at(row, from) : Row<DT>::empty();
    }
    __device__ __forceinline__ static int lead(const Row<DT> &row) { return row.first_full() + (int)__builtin_amdgcn_readfirstlane(threadIdx.x & ~63u); }
    __device__ __forceinline__ static int edge_slot(const Row<DT> &row)
    {
        if (threadIdx.x == 0 && row.shift) return 0;
        if (threadIdx.x == 1 && row.slots > row.end_full() && (row.slots > 1 || !row.shift)) return row.slots - 1;
        return -1;
    }
    __device__ __forceinline__ void fetch_edge(const Row<DT> &row)
    {
        const int s = edge_slot(row);
        edge = s >= 0 ? row.load(s) : Row<DT>::empty();
    }
    // f(raw) for the slots of the wavefront, held or read again; FIRST: those that LDS holds come from memory
    template <bool FIRST, typename F> __device__ __forceinline__ void each(const Row<DT> &row, F f) const
    {
        const int lead = this->lead(row), f0 = row.first_full(), f1 = row.end_full();
        if (threadIdx.x < 64) f(edge);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (lead + i * BLOCK < f1) f(v[i]);         // uniform for the wavefront
        auto more = [&](int i, auto keep) {             // slots i ... i + 3
            uint4 w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int s = f0 + (int)threadIdx.x + (i + k) * BLOCK;
                // what LDS keeps is read once; the rest is wanted again soon
                w[k] = s >= f1 ? Row<DT>::empty() : decltype(keep)::value ? load_at(row, f0 + (i + k) * BLOCK) : row.load_full(s);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (lead + (i + k) * BLOCK >= f1) break;
                f(w[k]);
                if constexpr (decltype(keep)::value) own[(i + k - NV) * BLOCK] = w[k];
            }
        };
        static_assert(NL % 4 == 0, "slots go in groups of four");
        if constexpr (NL > 0) {
            if constexpr (FIRST) {
#pragma unroll 1
                for (int i = NV; i < NV + NL && lead + i * BLOCK < f1; i += 4) more(i, std::true_type{});
            } else {
#pragma unroll 1
                for (int i = NV; i < NV + NL && lead + i * BLOCK < f1; ++i) f(own[(i - NV) * BLOCK]);
            }
        }
#pragma unroll 1
        for (int i = NV + NL; lead + i * BLOCK < f1; i += 4) more(i, std::false_type{});
    }
    __device__ __forceinline__ float4 sums(const Row<DT> &row, const Scales &q) const
    {
        auto largest = [&](float t, const uint4 &raw) {
            float x[VEC];
            Type::unpack(raw, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) t = fmaxf(t, x[j]);
            return t;
        };
        float t = -INFINITY;
        if (lead(row) < row.end_full()) t = largest(t, v[0]);
        if (threadIdx.x < 64) t = largest(t, edge);
        Reference<VEC> at(uniform(wave_max(t)), q);
        float s = 0.f, u = 0.f;
        each<true>(row, [&](const uint4 &raw) {
            float x[VEC];
            Type::unpack(raw, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float y = fmaf(x[j], at.c, -at.rc), e = exp2_fast(y);
                s += e;
                if constexpr (ENTROPY) u = fmaf(e, y, u);
            }
        });
        if (__any(!(at.ref > -INFINITY && s <= 0x1p12f && (!ENTROPY || fabsf(u) <= 0x1p30f)))) {
            float most = t;
            bool odd = false;
            each<false>(row, [&](const uint4 &raw) { most = largest(most, raw); });
            at.set(uniform(wave_max(most)), q);
            s = u = 0.f;
            if (at.ref > -INFINITY) {
                each<false>(row, [&](const uint4 &raw) {
                    float x[VEC];
                    Type::unpack(raw, x);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float y = at.by_difference() ? (x[j] - at.ref) * q.c : fmaf(x[j], at.c, -at.rc), e = exp2_fast(y);
                        s += e;
                        if constexpr (ENTROPY) u = fmaf(e, fmaxf(y, LEAST), u);
                    }
                });
            } else {
                each<false>(row, [&](const uint4 &raw) {
                    float x[VEC];
                    Type::unpack(raw, x);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) odd = odd || isnan(x[j]);
                });
                return make_float4(-INFINITY, __any(odd) ? NAN : 0.f, 0.f, 0.f);
            }
        }
        const float f = exp2_fast(-at.lost), ws = wave_sum(s), wu = ENTROPY ? wave_sum(u) : 0.f;
        return make_float4(at.ref, ws * f, ENTROPY ? f * fmaf(-at.lost, ws, wu) : 0.f, 0.f);
    }
};

template <int DT, int BLOCK, int NV, int NL, bool ENTROPY>
__global__ __launch_bounds__(BLOCK, NL > 0 ? 4 : 5) void token_loss_rows_kernel(ScoreArgs a)
{
    using Type = LogitType<DT>;
    constexpr int VEC = Type::VEC;
    __shared__ JoinLds<BLOCK> lds;
    __shared__ uint4 rest[NL > 0 ? NL * BLOCK : 1];
    const Scales q(a.temperature);
    const size_t r = blockIdx.x;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const GradRow<DT> out(a.dlogits, a.dld, a.V, r, row);
    const int token = a.tokens[r];
    if (padded(a, token)) {
        out.clear(row.slots, BLOCK);
        if (threadIdx.x == 0) write_score(a, r, true, false, make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0);
        return;
    }
    HeldRow<DT, BLOCK, NV, NL, ENTROPY> held;
    held.own = rest + threadIdx.x;
#pragma unroll
    for (int i = 0; i < NV; ++i) held.fetch(row, i);
    held.fetch_edge(row);
    const float z_token = row.load_one(token);
    const float4 w = join_waves<BLOCK>(held.sums(row, q), lds, q);
    const TokenSlope<VEC> g(a, r, false, w.x, w.y, w.z / w.y, z_token, q);
    if (g.none) {                                   // uniform
        out.clear(row.slots, BLOCK);
        if (threadIdx.x == 0) write_score(a, r, false, true, w, z_token, 0);
        return;
    }
    const TokenPlace<DT> place(row, token, g.of_token);
    if (g.at.by_difference() || !out.same) {        // uniform, and rare (large logits, a gradient at another alignment): the row is read again
#pragma unroll 1
        for (int s = threadIdx.x; s < row.slots; s += BLOCK) {
            float x[VEC];
            Type::unpack(row.load(s), x);
            if (g.at.by_difference()) g.of_difference(x, q);
            else g.template of<ENTROPY>(x);
            place.put(x, s);
            out.store(s, x, row.full(s));
        }
        if (threadIdx.x == 0) write_score(a, r, false, true, w, z_token, 0);
        return;
    }
    const int f0 = row.first_full(), f1 = row.end_full(), lead = held.lead(row), edge_slot = held.edge_slot(row);
    if (edge_slot >= 0) {
        float x[VEC];
        Type::unpack(held.edge, x);
        g.template of<ENTROPY>(x);
        place.put(x, edge_slot);
        out.store(edge_slot, x, false);
    }
    // full slots f0 + i * BLOCK + thread
    auto put = [&](const uint4 &raw, int i) {
        float x[VEC];
        Type::unpack(raw, x);
        g.template of<ENTROPY>(x);
        if ((unsigned)(place.slot - (lead + i * BLOCK)) < 64u) place.put(x, f0 + i * BLOCK + (int)threadIdx.x);        // uniform for the wavefront
        out.store_at(f0 + i * BLOCK, x);
    };
    if constexpr (NL > 0) {
#pragma unroll 2
        for (int i = NV; i < NV + NL; ++i)
            if (f0 + (int)threadIdx.x + i * BLOCK < f1) put(held.own[(i - NV) * BLOCK], i);
    }
#pragma unroll 1
    for (int i = NV + NL; lead + i * BLOCK < f1; i += 4) {
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (f0 + (int)threadIdx.x + (i + k) * BLOCK < f1) v[k] = row.load_full(f0 + (int)threadIdx.x + (i + k) * BLOCK);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (f0 + (int)threadIdx.x + (i + k) * BLOCK < f1) put(v[k], i + k);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (f0 + (int)threadIdx.x + i * BLOCK < f1) put(held.v[i], i);
    if (threadIdx.x == 0) write_score(a, r, false, true, w, z_token, 0);        // 64 bits, where no row is held any more
}

// ---- short rows: a wavefront each, all calls --------------------------------------------------------------------------------------
// Rows of at most 64 * NQ logits sit in a wavefront's registers, element lane + 64 i in x[i]; maximum, sums and counts are shuffles and
// votes, and nothing waits for other wavefronts.  Bound: latency.  2048 x 100 fp32, gradient: 3.6 us.
enum { SCORE_SUMS = 1, SCORE_GRAD = 2, SCORE_BOTH = 3 };
template <int DT, int NQ, int MODE, bool TOP>
__global__ __launch_bounds__(256) void score_short_kernel(ScoreArgs a)
{
    __shared__ unsigned long long all_words[TOP ? 4 : 1][TOP ? LOGITS_MAX_TOP : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t r = (size_t)blockIdx.x * 4 + wave;
    if (r >= a.rows) return;                            // wavefronts of a block have nothing in common
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const Scales q(a.temperature);
    const int token = a.tokens ? a.tokens[r] : -1;
    const bool padding = padded(a, token), given = a.tokens && !padding;
    float x[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int j = lane + 64 * i;
        x[i] = -INFINITY;
        if (j < a.V && !padding) {
            x[i] = row.load_one(j);
            if constexpr (DT == EASGD_F32)              // logits that come as partial sums: added in ascending order
                for (int p = 1; p < a.parts; ++p) x[i] += row.base[row.shift + j + p * a.part_stride];
        }
    }
    float z_token = 0.f;
    if (given) {                                        // uniform
        float z = x[0];
#pragma unroll
        for (int i = 1; i < NQ; ++i) z = token >> 6 == i ? x[i] : z;
        z_token = __shfl(z, token & 63);
    }
    float4 w = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if constexpr (MODE & SCORE_SUMS) {
        float m = x[0];
#pragma unroll
        for (int i = 1; i < NQ; ++i) m = fmaxf(m, x[i]);
        w.x = wave_max(m);
    } else {
        w = a.state[r];
    }
    const float from = w.x == -INFINITY ? 0.f : w.x;
    float y[NQ], e[NQ], s = 0.f, u = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        y[i] = (x[i] - from) * q.c;
        e[i] = exp2_fast(y[i]);
        y[i] = fmaxf(y[i], LEAST);
        s += e[i];
        u = fmaf(e[i], y[i], u);
    }
    float mean = 0.f;
    if constexpr (!(MODE & SCORE_SUMS)) mean = mean_exponent(w.y, w.z);
    if constexpr (MODE & SCORE_SUMS) {
        w.y = wave_sum(s);
        w.z = wave_sum(u);
        unsigned before = 0;
        if (a.rank && given) {
            const bool masked = !(z_token > -INFINITY);
#pragma unroll
            for (int i = 0; i < NQ; ++i)
                before += __popcll(__ballot(masked ? x[i] > -INFINITY : x[i] > z_token || (x[i] == z_token && lane + 64 * i < token)));
        }
        if (lane == 0) write_score(a, r, padding, given, w, z_token, before);
        mean = w.z / w.y;
        if constexpr (TOP) {
            const RowScore score(w);
            unsigned long long *words = all_words[wave];
            const unsigned n = short_first(x, (unsigned)a.k, words);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");         // LDS accesses of one wavefront are executed in order
            for (unsigned i = lane; i < (unsigned)a.k; i += 64) {
                unsigned at = i;
                if (i < n) {
                    at = 0;
                    for (unsigned j = 0; j < n; ++j) at += words[j] > words[i];
                }
                write_alternative(a, r, at, i < n ? words[i] : 0, score, w.x);
            }
        }
    }
    if constexpr (MODE & SCORE_GRAD) {
        const TokenSlope<4> g(a, r, padding, from, w.y, mean, z_token, q, true);
        const Row<DT> out(a.dlogits, r, a.dld, a.V);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int j = lane + 64 * i;
            const float d = g.none ? 0.f : j == token ? g.of_token : e[i] * fmaf(g.b, y[i], g.a);
            if (j < a.V) out.base[out.shift + j] = LogitType<DT>::narrow(d);
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------------------------------
// Into how many parts rows are cut: enough blocks to fill the chip, and at least 1024 slots (four per thread) a part.
static constexpr int SCORE_BLOCK = 256, SCORE_SPLIT_ROWS = 256, SCORE_SPLIT_BLOCKS = 1024, SCORE_SPLIT_SLOTS = 1024;
static int score_segments(size_t rows, int slots)
{
    if (rows >= SCORE_SPLIT_ROWS || slots < 2 * SCORE_SPLIT_SLOTS) return 1;
    const int want = (int)((SCORE_SPLIT_BLOCKS + rows - 1) / rows), most = slots / SCORE_SPLIT_SLOTS;
    return want < most ? want : most;
}
// Gradients of rows whose sums are there: parts of at least 1024 slots, 2048 blocks (1024 x 32000 bf16 22.3 us, with 1024 blocks 26.3; 777 x 50001 28.5
// and 34)
static constexpr int GRAD_BLOCKS = 2048;
static int grad_segments(size_t rows, int slots)
{
    const size_t want = (GRAD_BLOCKS + rows - 1) / rows, most = (size_t)slots / SCORE_SPLIT_SLOTS;
    return (int)(most < 1 ? 1 : want < most ? want : most);
}
static void set_segments(ScoreArgs &a, int segments, int slots)
{
    a.segments = segments;
    a.seg_slots = (slots + segments - 1) / segments;
}
static size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

template <typename F> static void by_flag(bool flag, F f)
{
    if (flag) f(std::true_type{});
    else f(std::false_type{});
}

// Logits past the caches where there are more of them than these (256 MB) hold for both who wrote and who reads them next.  Freshly written logits, us, past the
// caches / through them: sums of 2048 x 131072 bf16 109 / 129, 4096 x 32000 53 / 65, 777 x 50001 22.5 / 20.6, 1024 x 32000 18.5 / 17.0; gradients
// 204 / 229, 93 / 115, 34 / 29.5, 29.9 / 25.0.
static bool read_once(size_t bytes) { return bytes > ((size_t)128 << 20); }
template <int DT> static void launch_sums(const ScoreArgs &a, bool entropy, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows * a.segments));
    by_flag(entropy, [&](auto h) {
        by_flag(a.rank, [&](auto rank) {
            by_flag(read_once(a.rows * a.V * sizeof(typename LogitType<DT>::Stored)), [&](auto once) {
                EASGD_LAUNCH((score_rows_kernel<DT, SCORE_BLOCK, decltype(h)::value, decltype(rank)::value, decltype(once)::value>), grid, dim3(SCORE_BLOCK), 0, s, a);
            });
        });
    });
    if (a.segments > 1) EASGD_LAUNCH((score_join_kernel<DT>), dim3((unsigned)a.rows), dim3(64), 0, s, a);
}
template <int DT> static void launch_top(const ScoreArgs &a, hipStream_t s)
{
    EASGD_LAUNCH((score_top_kernel<DT, TOP_BLOCK>), dim3((unsigned)(a.rows * a.segments)), dim3(TOP_BLOCK), 0, s, a);
    if (a.segments > 1 && a.segments * a.k <= 256) EASGD_LAUNCH((score_top_join_kernel<DT, 256>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
    else if (a.segments > 1) EASGD_LAUNCH((score_top_join_kernel<DT, TOP_BLOCK>), dim3((unsigned)a.rows), dim3(TOP_BLOCK), 0, s, a);
}
// 512 threads where a part has work for them, us (256 / 512): 2048 x 131072 bf16 209 / 203, 777 x 50001 fp16 25.7 / 25.3, 2000 x 10000 bf16 14.4 / 15.1,
// 500 x 9000 fp32 6.9 / 7.8
template <int DT> static void launch_grad(const ScoreArgs &a, bool entropy, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows * a.segments));
    by_flag(entropy, [&](auto h) {
        by_flag(read_once(a.rows * a.V * sizeof(typename LogitType<DT>::Stored)), [&](auto once) {
            if (a.seg_slots >= 2048) EASGD_LAUNCH((score_grad_kernel<DT, 512, decltype(h)::value, decltype(once)::value>), grid, dim3(512), 0, s, a);
            else EASGD_LAUNCH((score_grad_kernel<DT, 256, decltype(h)::value, decltype(once)::value>), grid, dim3(256), 0, s, a);
        });
    });
}
template <int DT, int BLOCK, int NV, int NL> static void launch_held(const ScoreArgs &a, bool entropy, hipStream_t s)
{
    by_flag(entropy, [&](auto h) {
        EASGD_LAUNCH((token_loss_rows_kernel<DT, BLOCK, NV, NL, decltype(h)::value>), dim3((unsigned)a.rows), dim3(BLOCK), 0, s, a);
    });
}
// What is held where, us (the block's threads / slots a thread in registers / in LDS):
//   2048 x 131072 bf16   512/16/8 228   1024/4/8 229   1024/8/8 234   512/8/8 239
//   4096 x 32000 bf16    256/8/8 108    256/12/4 106   256/4/8 119    256/12/0 129
//   777 x 50001 fp16     256/8/8 34     256/12/4 36.5  256/4/8 35.5   256/12/0 39
template <int DT> static void launch_loss(const ScoreArgs &a, int slots, bool entropy, hipStream_t s)
{
    if (slots <= 2048) launch_held<DT, 256, 4, 0>(a, entropy, s);
    else if (slots <= 8192 + 2) launch_held<DT, 256, 8, 8>(a, entropy, s);
    else launch_held<DT, 512, 16, 8>(a, entropy, s);
}
template <int DT, int MODE, bool TOP> static void launch_short(const ScoreArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.rows + 3) / 4));
    if (a.V <= 128) EASGD_LAUNCH((score_short_kernel<DT, 2, MODE, TOP>), grid, dim3(256), 0, s, a);
    else EASGD_LAUNCH((score_short_kernel<DT, SCORE_SHORT_V / 64, MODE, TOP>), grid, dim3(256), 0, s, a);
}

int check_tokens(const char *name, const TokensGiven &t, bool rows)
{
    if (int rc = check_temperature(name, t.temperature)) return rc;
    if (!std::isfinite(t.bonus)) return fail(EASGD_EINVAL, "%s: bonus must be finite", name);
    if (rows && !t.tokens) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(t.tokens, 4) || !aligned_to(t.weight, 4) || !aligned_to(t.logprob, 4) || !aligned_to(t.entropy, 4))
        return fail(EASGD_EINVAL, "%s: tokens, weight, logprob, entropy must be 4-byte aligned", name);
    return EASGD_OK;
}

void score_logits(const float *logits, int parts, size_t part_stride, size_t rows, int classes, const TokensGiven &t, float scale,
                  float *row_loss, float *dlogits, void *stream)
{
    ScoreArgs a = {};
    a.logits = logits; a.ld = (size_t)classes; a.rows = rows; a.V = classes;
    a.tokens = t.tokens; a.temperature = t.temperature; a.weight = t.weight; a.bonus = t.bonus;
    a.logprob = t.logprob; a.entropy = t.entropy; a.loss = row_loss;
    a.scale = scale; a.dlogits = dlogits; a.dld = (size_t)classes; a.parts = parts; a.part_stride = part_stride; a.segments = 1;
    launch_short<EASGD_F32, SCORE_BOTH, false>(a, static_cast<hipStream_t>(stream));
}

}  // namespace easgd

extern "C" {

size_t easgd_score_tokens_workspace_bytes(size_t rows, int V, int k)
{
    using namespace easgd;
    if (rows == 0 || rows > LOGITS_MAX_ROWS || V < 1 || V > LOGITS_MAX_V || k < 0 || k > LOGITS_MAX_TOP) return 0;
    const int slots = most_slots(EASGD_F32, V);         // fp32 rows have the most slots, and the most parts
    const int n = k ? top_segments(rows, slots, k) : score_segments(rows, slots);
    return n == 1 ? 0 : rounded(rows * n * (sizeof(float4) + (size_t)k * 8));
}

int easgd_score_tokens(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *tokens, float temperature,
                       float *logprob, float *entropy, int32_t *rank, int k, float *top_logprob, int32_t *top_indices, float *state,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_score_tokens";
    if (int rc = check_logits(name, logits, dtype, rows, V, ld)) return rc;
    if (int rc = check_temperature(name, temperature)) return rc;
    if (k < 0 || k > LOGITS_MAX_TOP) return fail(EASGD_EINVAL, "%s: k must be in [0, %d], got %d", name, LOGITS_MAX_TOP, k);
    if (!tokens && (logprob || rank)) return fail(EASGD_EINVAL, "%s: logprob and rank need tokens", name);
    if (rows > 0 && k > 0 && (!top_logprob || !top_indices)) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (rows > 0 && k == 0 && !logprob && !entropy && !rank && !state) return fail(EASGD_EINVAL, "%s: nothing is asked for", name);
    if (!aligned_to(tokens, 4) || !aligned_to(logprob, 4) || !aligned_to(entropy, 4) || !aligned_to(rank, 4) || !aligned_to(top_logprob, 4) || !aligned_to(top_indices, 4))
        return fail(EASGD_EINVAL, "%s: tokens, logprob, entropy, rank, top_logprob, top_indices must be 4-byte aligned", name);
    if (!aligned16(state)) return fail(EASGD_EINVAL, "%s: state must be 16-byte aligned", name);
    if (int rc = check_workspace(name, workspace, workspace_bytes, easgd_score_tokens_workspace_bytes(rows, V, k))) return rc;
    clear_error();
    if (rows == 0) return EASGD_OK;
    ScoreArgs a = {};
    a.logits = logits; a.ld = ld; a.rows = rows; a.V = V;
    a.tokens = tokens; a.temperature = temperature;
    a.logprob = logprob; a.entropy = entropy; a.rank = rank; a.state = reinterpret_cast<float4 *>(state);
    a.k = k; a.top_logprob = top_logprob; a.top_indices = top_indices; a.parts = 1;
    const int slots = most_slots(dtype, V);
    set_segments(a, k ? top_segments(rows, slots, k) : score_segments(rows, slots), slots);
    a.partial = static_cast<float4 *>(workspace);
    a.words = reinterpret_cast<unsigned long long *>(a.partial + rows * a.segments);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (V <= SCORE_SHORT_V) {
            if (k) launch_short<DT, SCORE_SUMS, true>(a, s);
            else launch_short<DT, SCORE_SUMS, false>(a, s);
        } else if (k) launch_top<DT>(a, s);
        else launch_sums<DT>(a, entropy || state, s);
    });
    return check_launch(name);
}

int easgd_score_tokens_grad(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *tokens, float temperature,
                            const float *state, const float *dlogprob, const float *dentropy, float scale, void *dlogits, size_t dld, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_score_tokens_grad";
    if (int rc = check_logits(name, logits, dtype, rows, V, ld)) return rc;
    if (int rc = check_temperature(name, temperature)) return rc;
    if (!tokens && dlogprob) return fail(EASGD_EINVAL, "%s: dlogprob needs tokens", name);
    if (rows > 0 && (!state || !dlogits || (!dlogprob && !dentropy))) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(tokens, 4) || !aligned_to(dlogprob, 4) || !aligned_to(dentropy, 4))
        return fail(EASGD_EINVAL, "%s: tokens, dlogprob, dentropy must be 4-byte aligned", name);
    if (!aligned16(state)) return fail(EASGD_EINVAL, "%s: state must be 16-byte aligned", name);
    if (int rc = check_gradient(name, dlogits, dtype, rows, V, dld, scale)) return rc;
    if (rows && rows_overlap(logits, ld, dlogits, dld, V, rows, dtype_bytes(dtype))) return fail(EASGD_EINVAL, "%s: dlogits must not overlap logits", name);
    clear_error();
    if (rows == 0) return EASGD_OK;
    ScoreArgs a = {};
    a.logits = logits; a.ld = ld; a.rows = rows; a.V = V;
    a.tokens = tokens; a.temperature = temperature; a.state = reinterpret_cast<float4 *>(const_cast<float *>(state));
    a.dlogprob = dlogprob; a.dentropy = dentropy; a.scale = scale; a.dlogits = dlogits; a.dld = dld; a.parts = 1;
    const int slots = most_slots(dtype, V);
    set_segments(a, grad_segments(rows, slots), slots);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (V <= SCORE_SHORT_V) launch_short<DT, SCORE_GRAD, false>(a, s);
        else launch_grad<DT>(a, dentropy, s);
    });
    return check_launch(name);
}

size_t easgd_token_loss_workspace_bytes(size_t rows, int V)
{
    using namespace easgd;
    if (rows == 0 || rows > LOGITS_MAX_ROWS || V <= SCORE_SHORT_V || V > LOGITS_MAX_V) return 0;
    const int n = score_segments(rows, most_slots(EASGD_F32, V));
    return n == 1 ? 0 : rounded(rows * (n + 1) * sizeof(float4));
}

int easgd_token_loss(const void *logits, int dtype, size_t rows, int V, size_t ld, const int32_t *tokens, const float *weight, float bonus,
                     float temperature, float scale, float *loss, float *logprob, float *entropy, void *dlogits, size_t dld,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_token_loss";
    if (int rc = check_logits(name, logits, dtype, rows, V, ld)) return rc;
    if (int rc = check_tokens(name, {tokens, weight, bonus, temperature, logprob, entropy}, rows > 0)) return rc;
    if (rows > 0 && (!loss || !dlogits)) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(loss, 4)) return fail(EASGD_EINVAL, "%s: loss must be 4-byte aligned", name);
    if (int rc = check_gradient(name, dlogits, dtype, rows, V, dld, scale)) return rc;
    if (int rc = check_workspace(name, workspace, workspace_bytes, easgd_token_loss_workspace_bytes(rows, V))) return rc;
    if (rows && rows_overlap(logits, ld, dlogits, dld, V, rows, dtype_bytes(dtype))) return fail(EASGD_EINVAL, "%s: dlogits must not overlap logits", name);
    clear_error();
    if (rows == 0) return EASGD_OK;
    ScoreArgs a = {};
    a.logits = logits; a.ld = ld; a.rows = rows; a.V = V;
    a.tokens = tokens; a.temperature = temperature; a.weight = weight; a.bonus = bonus;
    a.loss = loss; a.logprob = logprob; a.entropy = entropy; a.scale = scale; a.dlogits = dlogits; a.dld = dld; a.parts = 1;
    a.partial = static_cast<float4 *>(workspace);
    const int slots = most_slots(dtype, V);
    set_segments(a, score_segments(rows, slots), slots);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (V <= SCORE_SHORT_V) launch_short<DT, SCORE_BOTH, false>(a, s);
        else if (a.segments == 1) launch_loss<DT>(a, slots, entropy || bonus != 0.f, s);
        else {
            a.state = a.partial + rows * a.segments;
            launch_sums<DT>(a, entropy || bonus != 0.f, s);
            launch_grad<DT>(a, bonus != 0.f, s);
        }
    });
    return check_launch(name);
}

}  // extern "C"
