// easgd_top_logits: the k first logits of every row's order, and the row's log-sum-exp.
//
// One pass: the sums of exponentials (row_sums.h) and the first k (logits_select.h) ride on the same loads.  Bound: HBM for many
// long rows (each logit once), latency for few or short ones.
#include "logits.h"
#include "logits_select.h"
#include "row_sums.h"

namespace easgd {

struct TopArgs {
    const void *logits;
    size_t ld, rows;
    int V, k;
    float temperature;
    float *values;
    int *indices;
    float *lse;
    int segments, seg_slots;           // slots of a part of a row
    unsigned long long *words;         // [rows][segments][k]: the first k of every part (0: none left)
    float4 *partial;                   // [rows][segments]: its sums
};

__device__ __forceinline__ void write_top(const TopArgs &a, size_t r, unsigned at, unsigned long long word)
{
    a.values[r * a.k + at] = word ? key_logit((unsigned)(word >> 32)) : -INFINITY;
    a.indices[r * a.k + at] = word ? (int)~(unsigned)word : -1;
}
__device__ __forceinline__ void write_lse(const TopArgs &a, size_t r, const float4 &s)
{
    if (a.lse) a.lse[r] = s.x == INFINITY ? INFINITY : (float)((double)(s.x == -INFINITY ? 0.f : s.x) / (double)a.temperature + log((double)s.y));
}
// the n words at the front of the list; places that are left over
__device__ __forceinline__ void write_list(const TopArgs &a, size_t r, const unsigned long long *list, unsigned n)
{
    const unsigned i = threadIdx.x;
    if (i < (unsigned)a.k) write_top(a, r, i, i < n ? list[i] : 0);
}

// ---- a block per row, or per part of a row ------------------------------------------------------------------------------
// Measured: 2048 x 131072 bf16, k = 64, 166 us a call in a row of calls = 3.2 TB/s, 179 traced by itself; the vector ALUs are busy 66 % of
// it.  Of 127 instructions a wavefront for 64 slots some 50 to 60 are the sums' (the two passes of distill_rows_kernel, with the packing, take 118);
// the others are selection: in the first rounds most slots hold a logit above the floor, which sends the whole wavefront through
// mask, key and list for it, and the list is ranked at the end.
template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void top_rows_kernel(TopArgs a)
{
    constexpr int VEC = Row<DT>::VEC;
    __shared__ TopLds lds;
    __shared__ float4 part[BLOCK / 64];
    const size_t r = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const Row<DT> row(a.logits, r, a.ld, a.V);
    const Scales q(a.temperature);
    const int s0 = seg * a.seg_slots, s1 = min(s0 + a.seg_slots, row.slots);
    RowSums<VEC, false, HARD_PLAIN> acc(q);
    const unsigned n = first_of<DT, BLOCK>(row, s0, s1, (unsigned)a.k, lds, [&](const float (&x)[VEC], int) { acc.add(x, 0u); });
    const float4 sums = acc.template combine<BLOCK>(part);
    if (a.segments == 1) {
        if (threadIdx.x == 0) write_lse(a, r, sums);
        write_list(a, r, lds.list, n);
        return;
    }
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sums;
    if ((int)threadIdx.x < a.k) a.words[(size_t)blockIdx.x * a.k + threadIdx.x] = threadIdx.x < n ? lds.list[threadIdx.x] : 0;
}

// ---- the parts of a row together ------------------------------------------------------------------------------------------
// Bound: latency.  8 x 50001 fp16, k = 20: parts 12.3 us, this kernel 4.6; a block per row took 79 us with the digits' walk.
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void top_join_kernel(TopArgs a)
{
    __shared__ TopLds lds;
    const size_t r = blockIdx.x;
    const unsigned all = (unsigned)(a.segments * a.k);             // <= TOP_LIST
    if (threadIdx.x < 64) {                             // the parts' sums, a part per lane (and every 64th after it), in a fixed order
        const Scales q(a.temperature);
        float4 own = make_float4(-INFINITY, 0.f, 0.f, 0.f);
        for (int i = threadIdx.x; i < a.segments; i += 64) {
            const float4 p = a.partial[r * a.segments + i], w = own;
            own = make_float4(fmaxf(w.x, p.x), 0.f, 0.f, 0.f);
            RowSums<4, false, HARD_PLAIN>::join(own, w, q);
            RowSums<4, false, HARD_PLAIN>::join(own, p, q);
        }
        float4 s = make_float4(wave_max(own.x), 0.f, 0.f, 0.f);
        RowSums<4, false, HARD_PLAIN>::join(s, own, q);
        s.y = wave_sum(s.y);
        if (threadIdx.x == 0) write_lse(a, r, s);
    }
    if (threadIdx.x == 0) lds.n = all;
    for (unsigned i = threadIdx.x; i < all; i += BLOCK) lds.list[i] = a.words[r * all + i];
    __syncthreads();
    unsigned n = keep_from<BLOCK>(lds, all, FIRST_WORD);           // the words that are there
    if (n > 512) n = keep_from<BLOCK>(lds, n, select_nth<BLOCK>(EachListed{lds.list, n, BLOCK}, FIRST_WORD, a.k, lds.select));
    rank_list<BLOCK>(lds, n, a.k);
    write_list(a, r, lds.list, min(n, (unsigned)a.k));
}

// ---- short rows: a wavefront each ---------------------------------------------------------------------------------------------
// Element lane + 64 q sits in register q.  The k-th largest key is found bit by bit with votes; equal keys are taken by
// ascending index, which is the order of registers, then lanes.  Bound: the votes' latency.  2048 x 1000 fp32, k = 10: 10.8 us.
template <int DT, int NQ>
__global__ __launch_bounds__(256) void top_short_kernel(TopArgs a)
{
    __shared__ unsigned long long all_words[4][LOGITS_MAX_TOP];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t r = (size_t)blockIdx.x * 4 + wave;
    if (r >= a.rows) return;                            // wavefronts of a block have nothing in common
    unsigned long long *words = all_words[wave];
    const Row<DT> row(a.logits, r, a.ld, a.V);
    float x[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) x[q] = lane + 64 * q < a.V ? row.load_one(lane + 64 * q) : -INFINITY;

    unsigned key[NQ], there = 0;
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        key[q] = logit_key(x[q]);
        there += __popcll(__ballot(key[q] != 0));
        m = fmaxf(m, x[q]);
    }
    if (a.lse) {
        m = wave_max(m);
        const float c = Scales(a.temperature).c, from = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < NQ; ++q) sum += exp2_fast((x[q] - from) * c);
        sum = wave_sum(sum);
        if (lane == 0) write_lse(a, r, make_float4(m, sum, 0.f, 0.f));
    }
    const unsigned k = min((unsigned)a.k, there);
    unsigned least = 1, above = there;                  // `above` keys are >= least
    if (there > k) {
        least = 0;
        for (unsigned bit = 0x80000000u; bit && above != k; bit >>= 1) {
            const unsigned next = least | bit;
            unsigned n = 0;
#pragma unroll
            for (int q = 0; q < NQ; ++q) n += __popcll(__ballot(key[q] >= next));
            if (n >= k) {
                least = next;
                above = n;
            }
        }
    }
    // keys above `least`, then as many equal ones as are wanted
    unsigned equal_left = k;
    if (above != k) {
        unsigned n = 0;
#pragma unroll
        for (int q = 0; q < NQ; ++q) n += __popcll(__ballot(key[q] > least));
        equal_left = k - n;
    }
    unsigned n = 0;
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const unsigned long long equal = __ballot(key[q] == least && key[q] != 0);
        const bool take = key[q] > least || (key[q] == least && key[q] != 0 && (unsigned)__popcll(equal & below) < equal_left);
        equal_left -= min(equal_left, (unsigned)__popcll(equal));
        const unsigned long long taken = __ballot(take);
        if (take) words[n + __popcll(taken & below)] = order_word(key[q], lane + 64 * q);
        n += __popcll(taken);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");         // LDS accesses of one wavefront are executed in order
    for (unsigned i = lane; i < (unsigned)a.k; i += 64) {
        unsigned rank = i;
        if (i < n) {
            rank = 0;
            for (unsigned j = 0; j < n; ++j) rank += words[j] > words[i];
        }
        write_top(a, r, rank, i < n ? words[i] : 0);
    }
}

// Few long rows are cut into parts, so that there are blocks for the whole chip: each part's first k go through the workspace.
// Many rows take blocks of 256 threads, five of which a compute unit holds (2048 x 131072 bf16, k = 64: 168 us against 180 with 512);
// few rows, and more than 64 tokens (whose first floor wants many maxima), 512 (8 x 50001: 15.8 us against 18.5 with 256).  The change at
// 256 rows suits a thousand rows and more better than some hundred, which leave a compute unit one to three blocks (us; 512 threads: k = 128):
//   rows of 131072 bf16     255 (four parts each)   256    512    768    1024   2048
//   256 threads, k = 64     49 (512 threads)        65     71     77     88     166
//   512 threads, k = 128    65                      46     56     88     106    204
static constexpr int TOP_BLOCK = 512, TOP_SHORT_V = 1024;
static constexpr int TOP_SPLIT_ROWS = 256, TOP_SPLIT_SLOTS = 2048;
static int top_segments(size_t rows, int slots, int k)
{
    if (rows >= TOP_SPLIT_ROWS || slots < 2 * TOP_SPLIT_SLOTS) return 1;
    int n = (int)((512 + rows - 1) / rows);
    if (n > slots / TOP_SPLIT_SLOTS) n = slots / TOP_SPLIT_SLOTS;
    if (n > TOP_LIST / k) n = TOP_LIST / k;
    return n < 1 ? 1 : n;
}
static size_t top_bytes(size_t rows, int segments, int k)
{
    return segments == 1 ? 0 : (rows * segments * (sizeof(float4) + (size_t)k * 8) + 255) / 256 * 256;
}

}  // namespace easgd

extern "C" {

size_t easgd_top_logits_workspace_bytes(size_t rows, int V, int k)
{
    using namespace easgd;
    if (rows == 0 || rows > LOGITS_MAX_ROWS || V < 1 || V > LOGITS_MAX_V || k < 1 || k > LOGITS_MAX_TOP) return 0;
    return top_bytes(rows, top_segments(rows, most_slots(EASGD_F32, V), k), k);     // fp32 rows have the most slots
}

int easgd_top_logits(const void *logits, int dtype, size_t rows, int V, size_t ld, int k, float temperature,
                     float *values, int32_t *indices, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace easgd;
    const char *name = "easgd_top_logits";
    if (int rc = check_logits(name, logits, dtype, rows, V, ld)) return rc;
    if (k < 1 || k > LOGITS_MAX_TOP) return fail(EASGD_EINVAL, "%s: k must be in [1, %d], got %d", name, LOGITS_MAX_TOP, k);
    if (int rc = check_temperature(name, temperature)) return rc;
    if (rows > 0 && (!values || !indices)) return fail(EASGD_EINVAL, "%s: NULL pointer", name);
    if (!aligned_to(values, 4) || !aligned_to(indices, 4) || !aligned_to(lse, 4)) return fail(EASGD_EINVAL, "%s: values, indices, lse must be 4-byte aligned", name);
    const size_t need = easgd_top_logits_workspace_bytes(rows, V, k);
    if (int rc = check_workspace(name, workspace, workspace_bytes, need)) return rc;
    clear_error();
    if (rows == 0) return EASGD_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int slots = most_slots(dtype, V), segments = top_segments(rows, slots, k);
    TopArgs a = {logits, ld, rows, V, k, temperature, values, indices, lse, segments, (slots + segments - 1) / segments, nullptr, nullptr};
    a.partial = static_cast<float4 *>(workspace);
    a.words = reinterpret_cast<unsigned long long *>(a.partial + rows * segments);
    by_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (V <= 128) EASGD_LAUNCH((top_short_kernel<DT, 2>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
        else if (V <= TOP_SHORT_V) EASGD_LAUNCH((top_short_kernel<DT, TOP_SHORT_V / 64>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
        else if (segments == 1 && rows >= TOP_SPLIT_ROWS && k <= 64) EASGD_LAUNCH((top_rows_kernel<DT, 256>), dim3((unsigned)rows), dim3(256), 0, s, a);
        else EASGD_LAUNCH((top_rows_kernel<DT, TOP_BLOCK>), dim3((unsigned)(rows * segments)), dim3(TOP_BLOCK), 0, s, a);
    });
    if (V > TOP_SHORT_V && segments > 1) EASGD_LAUNCH((top_join_kernel<TOP_BLOCK>), dim3((unsigned)rows), dim3(TOP_BLOCK), 0, s, a);
    return check_launch(name);
}

}  // extern "C"
