// Finding a place in the order of a row of logits: the order word of its n-th token, or of the token at which the mass of
// the tokens before it reaches a target.  General and exact for every row (ties, masked places, constant rows).
#pragma once
#include "logits.h"

namespace easgd {

// Order words are walked down digit by digit, largest first: 32 bits of key, then the 20 index bits that differ.
// The digits' bins are counted in LDS; the bin in which the target falls is the next level's interval.
static constexpr int SELECT_BINS = 2048;
static constexpr int SELECT_LEVELS = 5;
__host__ __device__ static constexpr int select_shift(int level) { return level == 0 ? 53 : level == 1 ? 42 : level == 2 ? 32 : level == 3 ? 10 : 0; }
__host__ __device__ static constexpr int select_bits(int level) { return level < 2 ? 11 : 10; }

struct SelectLds {
    unsigned long long mass[SELECT_BINS];
    unsigned count[SELECT_BINS];
    unsigned long long part[16];
    unsigned long long above;      // mass (or tokens) before the chosen bin
    unsigned bin, bin_count;
};

// The bin, from the last (largest) one down, at which the running sum of the weights first reaches target - above.
// weight(bin) is read by one thread each.  Every thread returns with the block's choice in lds.bin, lds.above, lds.bin_count.
template <int BLOCK, bool MASS>
__device__ __forceinline__ void select_bin(SelectLds &lds, int bins, unsigned long long above, unsigned long long target)
{
    constexpr int PER = SELECT_BINS / BLOCK;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long w[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = bins - 1 - (tid * PER + i);
        w[i] = b < 0 ? 0ull : MASS ? lds.mass[b] : (unsigned long long)lds.count[b];
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

// The smallest order word of the shortest prefix of the row's order whose weights reach `target` (>= 1; the weights of all
// words >= floor must reach it).  MASS: the weight of an element is mass(x), else 1.  Only words >= floor count.
// Passes over the row: one per level, until the chosen bin holds one element, or (counting) all of it is in the prefix.
template <int DT, int BLOCK, bool MASS, typename F>
__device__ __forceinline__ unsigned long long select_word(const Row<DT> &row, unsigned long long floor, unsigned long long target,
                                                          SelectLds &lds, F mass)
{
    constexpr int VEC = Row<DT>::VEC;
    unsigned long long prefix = 0, above = 0;
#pragma unroll 1
    for (int level = 0; level < SELECT_LEVELS; ++level) {
        const int shift = select_shift(level), bits = select_bits(level), bins = 1 << bits;
        if (level == 3) prefix |= 0xfff00000ull;        // the index bits above the twentieth are all ones
        __syncthreads();
        for (int b = threadIdx.x; b < bins; b += BLOCK) {
            lds.count[b] = 0;
            if constexpr (MASS) lds.mass[b] = 0;
        }
        __syncthreads();
        for (int s = threadIdx.x; s < row.slots; s += BLOCK) {
            float x[VEC];
            Row<DT>::Type::unpack(row.load(s), x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const unsigned long long word = order_word(logit_key(x[i]), row.index(s, i));
                if (word >= FIRST_WORD && word >= floor && (level == 0 || ((word ^ prefix) >> (shift + bits)) == 0)) {
                    const unsigned b = (unsigned)(word >> shift) & (bins - 1);
                    atomicAdd(&lds.count[b], 1u);
                    if constexpr (MASS) atomicAdd(&lds.mass[b], mass(x[i]));
                }
            }
        }
        __syncthreads();
        select_bin<BLOCK, MASS>(lds, bins, above, target);
        prefix |= (unsigned long long)lds.bin << shift;
        above = lds.above;
        if (lds.bin_count == 1 || (!MASS && above + lds.bin_count == target)) break;
    }
    return prefix > floor ? prefix : floor;
}

}  // namespace easgd
