// Index arithmetic of the attention kernels that the host's compiler can check too.
#pragma once

#ifdef __CUDACC__
#define CR_HD __host__ __device__ __forceinline__
#else
#define CR_HD static inline
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
