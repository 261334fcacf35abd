// Index arithmetic of the attention and writing kernels that the host's compiler can check too.
#pragma once

#ifdef __CUDACC__
#define CR_HD __host__ __device__ __forceinline__
#define CR_HD_MEMBER __host__ __device__ __forceinline__
#else
#define CR_HD static inline
#define CR_HD_MEMBER
#endif

// CTAs that worked on a block, as k_attn_rows and k_attn_few mark them: the first and how many.  A CTA whose waits have
// given up leaves marks unset, which are then whatever the memory holds: none leads outside [0, ncta).
struct cr_cta_span {
    int first;
    unsigned n;
};
CR_HD cr_cta_span cr_marked_ctas(int first, int last, int ncta)
{
    first = first < 0 ? 0 : (first > ncta - 1 ? ncta - 1 : first);
    last = last < first ? first : (last > ncta - 1 ? ncta - 1 : last);
    return {first, (unsigned)(last - first) + 1u};
}

// Sequences hold up to 2^31 - 8 keys: what is rounded up or goes a tile further is unsigned, and keys are compared by
// their distances.
CR_HD unsigned cr_key_tiles(int keys, unsigned tile) { return ((unsigned)keys + tile - 1) / tile; }
// Tiles of a single token's block, whose keys below lo are counted elsewhere; one at least, which writes zeros where
// there are no keys.
CR_HD unsigned cr_few_tiles(int lo, int klen, unsigned tile)
{
    const unsigned end = cr_key_tiles(klen, tile), begin = (unsigned)lo / tile;
    return end > begin + 1 ? end - begin : 1;
}
// Which of the 16 keys from `key` on a sequence sees, [first, end) of it: none, all or some.
struct cr_keys16 {
    int first, end;
    CR_HD_MEMBER bool any() const { return end > 0 && first < 16; }
    CR_HD_MEMBER bool all() const { return end >= 16 && first <= 0; }
    CR_HD_MEMBER bool sees(int j) const { return j >= first && j < end; }
};
CR_HD cr_keys16 cr_seen16(int key, int lo, int klen) { return {lo - key, klen - key}; }

// Writing: steps of 2^log2 positions that rows are worked on in.  Entry i, whose tokens begin at cu, has the slots from
// cr_slot_of(cu, i) on: its m tokens touch at most m / 2^log2 + 2 steps, which the next entry's first slot leaves it.
CR_HD unsigned long long cr_slot_of(int cu, unsigned i, unsigned log2) { return ((unsigned)cu >> log2) + 2ull * i; }
// Positions [begin, end) of the k-th step that the last m of a row's len tokens touch; none where begin >= end.
// Positions may be negative (more tokens than the row has), but not on both sides of 0 in a step.
struct cr_positions {
    long long begin, end;
};
CR_HD cr_positions cr_slot_positions(long long len, int m, unsigned long long k, unsigned log2)
{
    const long long size = 1ll << log2, first = len - m, step = (first >> log2) + (long long)k;
    const long long begin = step * size, end = begin + size;
    return {begin < first ? first : begin, end > len ? len : end};
}
