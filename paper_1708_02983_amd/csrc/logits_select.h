// Finding the first tokens of the order of a row of logits.
#pragma once
#include "logits.h"

namespace easgd {

// ---- a place in the order, exactly and for every row (ties, masked places, constant rows) ----------------------------
// Order words are walked down digit by digit, largest first: 32 bits of key, then the 20 index bits that differ.
// The digits' bins are counted in LDS; the bin in which the target falls is the next level's interval.
static constexpr int SELECT_BINS = 2048;
static constexpr int SELECT_LEVELS = 5;
__host__ __device__ static constexpr int select_shift(int level) { return level == 0 ? 53 : level == 1 ? 42 : level == 2 ? 32 : level == 3 ? 10 : 0; }
__host__ __device__ static constexpr int select_bits(int level) { return level < 2 ? 11 : 10; }

template <bool MASS> struct SelectLds {
    unsigned count[SELECT_BINS];
    unsigned long long mass[MASS ? SELECT_BINS : 1];
    unsigned long long part[16];
    unsigned long long above;      // mass (or tokens) before the chosen bin
    unsigned bin, bin_count;
};

// The bin, from the last (largest) one down, at which the running sum of the weights first reaches target - above.
// Every thread returns with the block's choice in lds.bin, lds.above, lds.bin_count.
template <int BLOCK, bool BY_MASS, bool MASS>
__device__ __forceinline__ void select_bin(SelectLds<MASS> &lds, int bins, unsigned long long above, unsigned long long target)
{
    constexpr int PER = SELECT_BINS / BLOCK;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long w[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = bins - 1 - (tid * PER + i);
        w[i] = b < 0 ? 0ull : BY_MASS ? lds.mass[MASS ? b : 0] : (unsigned long long)lds.count[b];
        sum += w[i];
    }
    unsigned long long run = sum;                       // inclusive over the lanes
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long up = __shfl_up(run, o);
        if (lane >= o) run += up;
    }
    if (lane == 63) lds.part[wave] = run;
    __syncthreads();
    unsigned long long before = above + run - sum;
    for (int v = 0; v < wave; ++v) before += lds.part[v];
    if (before < target && before + sum >= target) {    // one thread: the running sums ascend
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (before < target && before + w[i] >= target) {
                const int b = bins - 1 - (tid * PER + i);
                lds.bin = (unsigned)b;
                lds.above = before;
                lds.bin_count = lds.count[b];
            }
            before += w[i];
        }
    }
    __syncthreads();
}

// The smallest order word of the shortest prefix of the order whose weights reach `target` (>= 1; the weights of all words
// >= floor must reach it).  each(f) calls f(word, logit) for every element (or order word) there is, through the threads
// of the block; words below `floor` do not count.  BY_MASS: the weight of an element is mass(logit), else 1.
// Calls of each: one per level, until the chosen bin holds one element, or (counting) all of it is in the prefix.
template <int BLOCK, bool BY_MASS, bool MASS, typename E, typename F>
__device__ __forceinline__ unsigned long long select_word(E each, unsigned long long floor, unsigned long long target, SelectLds<MASS> &lds, F mass)
{
    unsigned long long prefix = 0, above = 0;
#pragma unroll 1
    for (int level = 0; level < SELECT_LEVELS; ++level) {
        const int shift = select_shift(level), bits = select_bits(level), bins = 1 << bits;
        if (level == 3) prefix |= 0xfff00000ull;        // the index bits above the twentieth are all ones
        __syncthreads();
        for (int b = threadIdx.x; b < bins; b += BLOCK) {
            lds.count[b] = 0;
            if constexpr (BY_MASS) lds.mass[b] = 0;
        }
        __syncthreads();
        each([&](unsigned long long word, float x) {
            if (word >= FIRST_WORD && word >= floor && (level == 0 || ((word ^ prefix) >> (shift + bits)) == 0)) {
                const unsigned b = (unsigned)(word >> shift) & (bins - 1);
                atomicAdd(&lds.count[b], 1u);
                if constexpr (BY_MASS) atomicAdd(&lds.mass[b], mass(x));
            }
        });
        __syncthreads();
        select_bin<BLOCK, BY_MASS>(lds, bins, above, target);
        prefix |= (unsigned long long)lds.bin << shift;
        above = lds.above;
        if (lds.bin_count == 1 || (!BY_MASS && above + lds.bin_count == target)) break;
    }
    __syncthreads();
    return prefix > floor ? prefix : floor;
}
template <int BLOCK, bool MASS, typename E>
__device__ __forceinline__ unsigned long long select_nth(E each, unsigned long long floor, unsigned n, SelectLds<MASS> &lds)
{
    return select_word<BLOCK, false>(each, floor, (unsigned long long)n, lds, [](float) { return 0ull; });
}

// Every slot of [s0, s1) through the threads of a block, eight loads under way at a time: f(raw, slot).
template <int DT, int BLOCK, typename F> __device__ __forceinline__ void each_slot(const Row<DT> &row, int s0, int s1, F f)
{
    constexpr int DEEP = 8;
    for (int s = s0 + (int)threadIdx.x; s < s1; s += DEEP * BLOCK) {
        uint4 v[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if (s + i * BLOCK < s1) v[i] = row.load_wave(s + i * BLOCK, s1);
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if (s + i * BLOCK < s1) f(v[i], s + i * BLOCK);
    }
}

// the elements of slots [s0, s1) of a row, as select_word takes them
template <int DT, int BLOCK> struct EachElement {
    const Row<DT> &row;
    int s0, s1;
    template <typename F> __device__ __forceinline__ void operator()(F f) const
    {
        each_slot<DT, BLOCK>(row, s0, s1, [&](const uint4 &raw, int s) {
            float x[Row<DT>::VEC];
            Row<DT>::Type::unpack(raw, x);
#pragma unroll
            for (int i = 0; i < Row<DT>::VEC; ++i) f(order_word(logit_key(x[i]), row.index(s, i)), x[i]);
        });
    }
};

// ---- the first k of the order in one pass -----------------------------------------------------------------------------
// A list in LDS takes every element above a floor that rises as the row goes by: first to the k-th largest of the threads'
// maxima over the first round of slots (k of them are at least as large, so the k-th of the row is), then, whenever the
// list has grown, to the k-th of the list.  On average a round adds k over the number of rounds gone by, so the list stays
// short and the loop over the row has one maximum and one comparison per 128 bits.  Rows that overflow the list all the
// same (ascending ones, more ties than it holds) are walked down digit by digit instead.
static constexpr int TOP_LIST = 2048;
struct TopLds {
    unsigned long long list[TOP_LIST];
    unsigned n;
    SelectLds<false> select;
};
struct EachListed {
    const unsigned long long *list;
    unsigned n;
    int block;
    template <typename F> __device__ __forceinline__ void operator()(F f) const
    {
        for (unsigned i = threadIdx.x; i < n; i += block) f(list[i], 0.f);
    }
};

// the list's words from `floor` on to its front; returns their number.  Ends with a barrier.
template <int BLOCK> __device__ __forceinline__ unsigned keep_from(TopLds &lds, unsigned n, unsigned long long floor)
{
    constexpr int PER = TOP_LIST / BLOCK;
    unsigned long long w[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned at = threadIdx.x + i * BLOCK;
        w[i] = at < n ? lds.list[at] : 0;
    }
    __syncthreads();
    if (threadIdx.x == 0) lds.n = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (w[i] >= FIRST_WORD && w[i] >= floor) lds.list[atomicAdd(&lds.n, 1u)] = w[i];
    __syncthreads();
    return lds.n;
}

// The list's n words in the order, at its front: every word's rank is the number of larger ones.  n <= 2 * BLOCK; only the first
// k are wanted.  Ends with a barrier.
template <int BLOCK> __device__ __forceinline__ void rank_list(TopLds &lds, unsigned n, unsigned k)
{
    const unsigned i = threadIdx.x, j = i + BLOCK;
    const unsigned long long one = i < n ? lds.list[i] : 0, two = j < n ? lds.list[j] : 0;
    unsigned rank_one = 0, rank_two = 0;
    if (n <= BLOCK) {                                   // uniform
#pragma unroll 4
        for (unsigned q = 0; q < n; ++q) rank_one += lds.list[q] > one;
    } else {
#pragma unroll 4
        for (unsigned q = 0; q < n; ++q) {
            const unsigned long long w = lds.list[q];
            rank_one += w > one;
            rank_two += w > two;
        }
    }
    __syncthreads();
    if (i < n && rank_one < k) lds.list[rank_one] = one;
    if (j < n && rank_two < k) lds.list[rank_two] = two;
    __syncthreads();
}

// A floor that at least k of the threads' logits t reach (k <= number of threads with t > -inf), a little below the k-th largest:
// the lower edge of its bin among 2048 of equal width between the smallest and the largest t.  lds.select is scratch.
template <int BLOCK> __device__ __forceinline__ float floor_of(float t, unsigned k, TopLds &lds)
{
    float *part = reinterpret_cast<float *>(lds.select.part);
    const float top = block_max<BLOCK>(t, part), bottom = -block_max<BLOCK>(t > -INFINITY ? -t : -INFINITY, part);
    // halves: the range of all finite logits fits
    const float range = top * 0.5f - bottom * 0.5f;
    if (!(range > 0.f) || range == INFINITY) return bottom;
    const float width = (float)(SELECT_BINS - 1) / range;
    for (int b = threadIdx.x; b < SELECT_BINS; b += BLOCK) lds.select.count[b] = 0;
    __syncthreads();
    if (t > -INFINITY) atomicAdd(&lds.select.count[(int)fminf((t * 0.5f - bottom * 0.5f) * width, (float)(SELECT_BINS - 1))], 1u);
    __syncthreads();
    select_bin<BLOCK, false>(lds.select, SELECT_BINS, 0, k);
    const float edge = ((float)lds.select.bin / width + bottom * 0.5f) * 2.f, room = (fabsf(top) + fabsf(bottom)) * 1e-6f;
    return width < INFINITY && edge - room > bottom ? edge - room : bottom;
}

// The order words of the first k (<= LOGITS_MAX_TOP) elements of slots [s0, s1), in the order, at the front of lds.list; returns
// how many there are (fewer than k where fewer are above -inf).  seen(x, slot) is called for every slot by whole wavefronts
// (an empty slot where a lane has none).  Ends with a barrier.
//
// One pass.  The maxima of BLOCK threads over their first slots are logits of the row, so the k-th largest of them is at most
// the k-th largest logit: a floor that leaves a few hundred of 131072 logits, found with one pass over bins in LDS.  What
// reaches the floor goes to a list in LDS, and the floor rises to the list's k-th word whenever the list has grown.  A row that
// overruns the list (ascending logits, many equal ones) is walked digit by digit instead.  (2048 x 131072 bf16, k = 64: 826 us
// with that walk for every row, five passes; 167 this way.)
template <int DT, int BLOCK, typename F>
__device__ __forceinline__ unsigned first_of(const Row<DT> &row, int s0, int s1, unsigned k, TopLds &lds, F seen)
{
    constexpr int VEC = Row<DT>::VEC, DEEP = 4;
    static_assert(BLOCK >= LOGITS_MAX_TOP && TOP_LIST % BLOCK == 0, "one maximum per thread has to do for the first floor");
    using Type = typename Row<DT>::Type;
    const int tid = threadIdx.x;
    const unsigned grown = max(4 * k, 256u);            // words after which the floor is raised again
    uint4 v[DEEP];
#pragma unroll
    for (int i = 0; i < DEEP; ++i) v[i] = row.load_wave(s0 + tid + i * BLOCK, s1);
    unsigned long long floor = FIRST_WORD;
    if (tid == 0) lds.n = 0;
    if ((s1 - s0) * VEC > TOP_LIST / 4) {
        float t = -INFINITY;
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            float x[VEC];
            Type::unpack(v[i], x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) t = fmaxf(t, x[j]);
        }
        if ((unsigned)__syncthreads_count(t > -INFINITY) >= k) floor = order_word(logit_key(floor_of<BLOCK>(t, k, lds)), -1);
    }
    __syncthreads();
    float least = 0.f;                                  // the floor as a logit; every logit that may be taken is at least -FLT_MAX
    auto set_least = [&]() { least = key_logit(max((unsigned)(floor >> 32), 0x00800000u)); };
    set_least();
    unsigned n = 0;
    bool over = false;
    for (int s = s0 + tid;;) {
        const int now = s;
        s += DEEP * BLOCK;
        const bool more = s - tid < s1;                 // uniform
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const int at = now + i * BLOCK, ahead = s + i * BLOCK;
            if (at - (tid & 63) >= s1) break;           // the whole wavefront is behind the end
            float x[VEC];
            Type::unpack(v[i], x);
            seen(x, at);
            float t = x[0];
#pragma unroll
            for (int j = 1; j < VEC; ++j) t = fmaxf(t, x[j]);
            if (!over && __any(t >= least)) {           // uniform for the wavefront
                // a bit per element, the last one's lowest; nearly always a few lanes have one
                unsigned hits = 0;
#pragma unroll
                for (int j = 0; j < VEC; ++j) hits = hits + hits + (x[j] >= least ? 1u : 0u);
                while (hits) {
                    const int j = VEC - __ffs(hits);
                    hits &= hits - 1;
                    const unsigned long long word = order_word(logit_key(Type::pick(v[i], j)), row.index(at, j));
                    if (word >= floor) {
                        const unsigned to = atomicAdd(&lds.n, 1u);
                        if (to < TOP_LIST) lds.list[to] = word;
                    }
                }
            }
            if (more) v[i] = row.load_wave(ahead, s1);  // the next round's slot
        }
        if (!more) break;
        __syncthreads();
        n = lds.n;
        over = over || n > TOP_LIST;                    // uniform
        if (!over && n > grown) {
            floor = select_nth<BLOCK>(EachListed{lds.list, n, BLOCK}, floor, k, lds.select);
            keep_from<BLOCK>(lds, n, floor);
            set_least();
        } else __syncthreads();                         // everyone has read n before it grows again
    }
    __syncthreads();
    n = lds.n;
    over = over || n > TOP_LIST;
    if (over) {
        // k elements are above the floor: its first value came from k maxima, later ones from k listed words
        floor = select_nth<BLOCK>(EachElement<DT, BLOCK>{row, s0, s1}, FIRST_WORD, k, lds.select);
        if (tid == 0) lds.n = 0;
        __syncthreads();
        EachElement<DT, BLOCK>{row, s0, s1}([&](unsigned long long word, float) {
            if (word >= floor && word >= FIRST_WORD) {
                const unsigned to = atomicAdd(&lds.n, 1u);
                if (to < TOP_LIST) lds.list[to] = word;         // always, unless the logits change under the kernel
            }
        });
        __syncthreads();
        n = min(lds.n, k);
    } else if (n > 512) {                               // more than a look at every pair is worth
        floor = select_nth<BLOCK>(EachListed{lds.list, n, BLOCK}, floor, k, lds.select);
        n = keep_from<BLOCK>(lds, n, floor);
    }
    rank_list<BLOCK>(lds, n, k);
    return min(n, k);
}

// The order words of the first k elements of a row that a wavefront holds, element lane + 64 q in x[q] (-inf behind the row's end),
// into words, in no order; returns how many there are.  The k-th largest key is found bit by bit with votes; equal keys are taken by
// ascending index, which is the order of registers, then lanes.
template <int NQ> __device__ __forceinline__ unsigned short_first(const float (&x)[NQ], unsigned k, unsigned long long *words)
{
    unsigned key[NQ], there = 0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        key[q] = logit_key(x[q]);
        there += __popcll(__ballot(key[q] != 0));
    }
    k = min(k, there);
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
    const int lane = threadIdx.x & 63;
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
    return n;
}

// ---- launch shapes of the kernels that take the first k ----
// Few long rows are cut into parts, so that there are blocks for the whole chip: each part's first k go through the workspace.
// Many rows take blocks of 256 threads, five of which a compute unit holds (2048 x 131072 bf16, k = 64: 168 us against 180 with 512);
// few rows, and more than 64 tokens (whose first floor wants many maxima), 512 (8 x 50001: 15.8 us against 18.5 with 256).  The change at
// 256 rows suits a thousand rows and more better than some hundred, which leave a compute unit one to three blocks (us; 512 threads: k = 128):
//   rows of 131072 bf16     255 (four parts each)   256    512    768    1024   2048
//   256 threads, k = 64     49 (512 threads)        65     71     77     88     166
//   512 threads, k = 128    65                      46     56     88     106    204
static constexpr int TOP_BLOCK = 512, TOP_SHORT_V = 1024;
static constexpr int TOP_SPLIT_ROWS = 256, TOP_SPLIT_SLOTS = 2048;
static inline int top_segments(size_t rows, int slots, int k)
{
    if (rows >= TOP_SPLIT_ROWS || slots < 2 * TOP_SPLIT_SLOTS) return 1;
    int n = (int)((512 + rows - 1) / rows);
    if (n > slots / TOP_SPLIT_SLOTS) n = slots / TOP_SPLIT_SLOTS;
    if (n > TOP_LIST / k) n = TOP_LIST / k;
    return n < 1 ? 1 : n;
}

}  // namespace easgd
