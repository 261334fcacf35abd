// Pages of a destination's key/value cache (include/cacheroute.h): extend, fork, free, compact, and
// writing new tokens' keys and values.
//
// Pages hold 16-bit elements, or 8-bit ones with a scale for every block of tokens and head, which go where
// the page's data goes.
//
// A call that takes pages needs the k-th free page for many k at once.  k_pages_scan writes the free
// pages as a bitmap with counts per 32-page word (within its chunk) and per chunk; any thread of the
// next kernel then finds the page of a rank, or the rank of a page, by a search of the chunk counts
// (in shared memory) and of the chunk's words.  Both kernels read the counts of every page once
// (4 bytes a page) and are bound by their launches until the pool has millions of pages; copies of
// page data are 16 bytes a thread with four loads in flight, bound by memory (664 MB of pages moved in
// 226 us, 6.0 TB/s; a thousand forks with tails of 8 tokens on average, 4 planes: 14 us with cold caches).
#include "cr_pages.cuh"

namespace {

constexpr uint32_t kMaxChunks = 1024;

// Scratch of one call.
struct pages_scan {
    uint32_t *bits;   // [words] free pages
    uint32_t *wpre;   // [words] free pages of the word's chunk before it
    uint32_t *cnt;    // [chunks] free pages
    uint32_t chunk_log2, chunks, n_pages;
    int4 *entry;      // [n] extend: (row, length, add, -); fork: (row, parent, keep, -); row < 0: skipped
    uint32_t *base;   // [n] pages taken by the entries before (saturated)
    unsigned long long *need;  // [1]
};

enum { SCAN_NONE, SCAN_EXTEND, SCAN_FORK };

template <typename T>
__device__ T block_scan(T v, T *total)  // exclusive, blockDim.x <= 1024
{
    __shared__ T part[32];
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
    T x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(~0u, x, o);
        if (lane >= (uint32_t)o) x += y;
    }
    if (lane == 31) part[w] = x;
    __syncthreads();
    if (w == 0) {
        T p = lane < nw ? part[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T y = __shfl_up_sync(~0u, p, o);
            if (lane >= (uint32_t)o) p += y;
        }
        part[lane] = p;
    }
    __syncthreads();
    const T before = w ? part[w - 1] : 0;
    *total = part[31];
    __syncthreads();
    return before + x - v;
}

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, uint32_t log2) { return (tokens + (1u << log2) - 1) >> log2; }

// Block 0: the entries' needs in list order.  The others: one chunk of pages each.
template <int KIND>
__global__ void __launch_bounds__(1024) k_pages_scan(const __grid_constant__ pages_in P, const __grid_constant__ pages_scan S,
                                                     const int32_t *a, const int32_t *b, const int32_t *c, uint32_t n)
{
    cr_launch_next();
    cr_wait_previous();
    if (KIND != SCAN_NONE && blockIdx.x == 0) {
        __shared__ int rows[1024];
        unsigned long long base = 0;
        for (uint32_t i0 = 0; i0 < n; i0 += 1024) {
            const uint32_t i = i0 + threadIdx.x;
            int4 e = make_int4(-1, 0, 0, 0);
            uint32_t need = 0;
            int row = -1, len = 0;  // an entry that can be carried out: its row, which has len tokens
            if (i < n) {
                if (KIND == SCAN_EXTEND) {
                    const int r = a[i], add = b[i];
                    if (r >= 0 && (uint32_t)r < P.n_seqs && add >= 0) {
                        len = __ldcg(P.lens + r);
                        if (len >= 0 && (long long)len + add <= ((long long)P.max_pages << P.page_log2)) {
                            row = r;
                            e = make_int4(r, len, add, 0);
                            need = pages_of((uint32_t)len + (uint32_t)add, P.page_log2) - pages_of((uint32_t)len, P.page_log2);
                        }
                    }
                } else {
                    const int src = a[i], dst = b[i], keep = c[i];
                    if (src >= 0 && (uint32_t)src < P.n_seqs && dst >= 0 && (uint32_t)dst < P.n_seqs && keep >= 1 &&
                        keep <= __ldcg(P.lens + src) && pages_of((uint32_t)keep, P.page_log2) <= P.max_pages &&
                        __ldcg(P.lens + dst) == 0) {
                        row = dst;
                        e = make_int4(dst, src, keep, 0);
                        need = (keep & (int)(P.page - 1)) != 0;
                    }
                }
            }
            __syncthreads();  // lengths are read before any is marked
            // A row is claimed (its length stands as -1 - len) by the entry that changes it: of several, the first in the
            // list.  Those of this round meet here; later ones find the mark.  The needs are summed while the claims are on
            // their way, in 64 bits: a row may ask for 2^28 pages.
            const int was = row >= 0 ? atomicCAS(P.lens + row, len, -1 - len) : len;
            unsigned long long total, at = block_scan((unsigned long long)need, &total);
            bool ok = row >= 0;
            if (__syncthreads_or(was != len)) {
                rows[threadIdx.x] = row;
                __syncthreads();
                for (uint32_t j = 0; ok && j < threadIdx.x; ++j) ok = rows[j] != row;
                at = block_scan(ok ? (unsigned long long)need : 0ull, &total);
            }
            at += base;
            if (!ok) {
                e.x = -1;
                if (i < n) atomicOr(P.status, CR_FLAG_BADPAGES);
            }
            if (i < n) {
                S.entry[i] = e;
                S.base[i] = at < 0xffffffffull ? (uint32_t)at : 0xffffffffu;
            }
            base += total;
        }
        if (threadIdx.x == 0) *S.need = base;
        return;
    }
    const uint32_t chunk = blockIdx.x - (KIND != SCAN_NONE), w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ uint32_t count[32];
    uint32_t before = 0;
    for (uint32_t r = 0; r < (1u << S.chunk_log2); r += 1024) {
        const uint64_t p = ((uint64_t)chunk << S.chunk_log2) + r + threadIdx.x;
        const bool free_page = p < P.n_pages && P.ref[p] == 0;
        const uint32_t word = __ballot_sync(~0u, free_page);
        if (lane == 0) count[w] = __popc(word);
        __syncthreads();
        uint32_t x = count[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(~0u, x, o);
            if (lane >= (uint32_t)o) x += y;
        }
        const uint32_t mine = before + (w ? __shfl_sync(~0u, x, w - 1) : 0);
        before += __shfl_sync(~0u, x, 31);
        if (lane == 0) {
            S.bits[p >> 5] = word;
            S.wpre[p >> 5] = mine;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) S.cnt[chunk] = before;
}

// Free pages before each chunk, into shared memory (every thread of the block calls it).
struct page_index {
    const uint32_t *pre;  // [chunks + 1]
    const pages_scan *S;
    __device__ void build(const pages_scan &s, uint32_t *smem)
    {
        S = &s;
        pre = smem;
        uint32_t base = 0;
        for (uint32_t i0 = 0; i0 < s.chunks; i0 += blockDim.x) {
            const uint32_t i = i0 + threadIdx.x;
            uint32_t total;
            const uint32_t at = base + block_scan(i < s.chunks ? s.cnt[i] : 0, &total);
            if (i < s.chunks) smem[i] = at;
            base += total;
        }
        if (threadIdx.x == 0) smem[s.chunks] = base;
        __syncthreads();
    }
    __device__ uint32_t free_pages() const { return pre[S->chunks]; }
    // free pages below p (p <= n_pages)
    __device__ uint32_t rank_free(uint32_t p) const
    {
        const uint32_t c = p >> S->chunk_log2;
        if (c >= S->chunks) return pre[S->chunks];
        return pre[c] + S->wpre[p >> 5] + __popc(S->bits[p >> 5] & ((1u << (p & 31)) - 1));
    }
    // the k-th bit of a word
    static __device__ __forceinline__ uint32_t bit_of(uint32_t word, uint32_t k)
    {
        uint32_t at = 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const uint32_t low = __popc(word & ((1u << o) - 1));
            if (k >= low) {
                k -= low;
                word >>= o;
                at += o;
            }
        }
        return at;
    }
    // last chunk with at most k free (LIVE: live) pages before it; k becomes the rank within it
    template <bool LIVE>
    __device__ __forceinline__ uint32_t chunk_of(uint32_t &k) const
    {
        uint32_t lo = 0, hi = S->chunks;
        while (hi - lo > 1) {
            const uint32_t m = (lo + hi) >> 1;
            if ((LIVE ? (m << S->chunk_log2) - pre[m] : pre[m]) <= k)
                lo = m;
            else
                hi = m;
        }
        k -= LIVE ? (lo << S->chunk_log2) - pre[lo] : pre[lo];
        return lo;
    }
    // The k-th free (LIVE: live) page, which exists, found by one thread.
    template <bool LIVE>
    __device__ uint32_t select(uint32_t k) const
    {
        const uint32_t w0 = chunk_of<LIVE>(k) << (S->chunk_log2 - 5);
        uint32_t a = 0, b = 1u << (S->chunk_log2 - 5);
        while (b - a > 1) {
            const uint32_t m = (a + b) >> 1;
            const uint32_t v = S->wpre[w0 + m];
            if ((LIVE ? 32 * m - v : v) <= k)
                a = m;
            else
                b = m;
        }
        const uint32_t v = S->wpre[w0 + a], word = S->bits[w0 + a];
        return ((w0 + a) << 5) + bit_of(LIVE ? ~word : word, k - (LIVE ? 32 * a - v : v));
    }
    // The same by a warp: 32 words at a look, one after the other only in pools of more than a million pages.
    template <bool LIVE>
    __device__ uint32_t select_warp(uint32_t k) const
    {
        const uint32_t lane = threadIdx.x & 31, w0 = chunk_of<LIVE>(k) << (S->chunk_log2 - 5);
        uint32_t at = 0, v = 0;
        for (uint32_t step = 1u << (S->chunk_log2 - 10);; step >>= 5) {
            if (step == 0) step = 1;
            const uint32_t m = at + lane * step, words = 1u << (S->chunk_log2 - 5);
            const bool in = m < words;
            v = in ? S->wpre[w0 + m] : 0;
            const uint32_t word = in ? S->bits[w0 + m] : 0;
            const uint32_t last = 31 - __clz(__ballot_sync(~0u, in && (LIVE ? 32 * m - v : v) <= k));
            at = __shfl_sync(~0u, m, last);
            if (step == 1) {
                v = __shfl_sync(~0u, v, last);
                const uint32_t w = __shfl_sync(~0u, word, last);
                return ((w0 + at) << 5) + bit_of(LIVE ? ~w : w, k - (LIVE ? 32 * at - v : v));
            }
        }
    }
};

// 16-byte words of one segment, four loads in flight.
__device__ __forceinline__ void copy16(uint4 *dst, const uint4 *src, uint32_t words)
{
    uint32_t i = threadIdx.x;
    for (; i + 3 * blockDim.x < words; i += 4 * blockDim.x) {
        const uint4 a = __ldcs(src + i), b = __ldcs(src + i + blockDim.x), c = __ldcs(src + i + 2 * blockDim.x),
                    d = __ldcs(src + i + 3 * blockDim.x);
        dst[i] = a;
        dst[i + blockDim.x] = b;
        dst[i + 2 * blockDim.x] = c;
        dst[i + 3 * blockDim.x] = d;
    }
    for (; i < words; i += blockDim.x) dst[i] = src[i];
}

// A block per entry: its pages, a warp each where they are few, else a thread.
__global__ void __launch_bounds__(128) k_pages_extend(const __grid_constant__ pages_in P, const __grid_constant__ pages_scan S,
                                                      uint32_t n)
{
    cr_launch_next();
    cr_wait_previous();
    __shared__ uint32_t pre[kMaxChunks + 1];
    page_index I;
    I.build(S, pre);
    const unsigned long long need = *S.need;
    const bool ok = need <= I.free_pages();
    if (!ok && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(P.status, CR_FLAG_NOPAGES);
    const int4 e = S.entry[blockIdx.x];
    if (e.x < 0) return;
    if (threadIdx.x == 0) P.lens[e.x] = ok ? e.y + e.z : e.y;
    if (!ok) return;
    const uint32_t had = pages_of((uint32_t)e.y, P.page_log2), now = pages_of((uint32_t)(e.y + e.z), P.page_log2);
    int32_t *row = P.table + (uint64_t)e.x * P.max_pages;
    const uint32_t first = S.base[blockIdx.x];
    if (now - had <= 8) {  // a warp a page
        for (uint32_t j = had + (threadIdx.x >> 5); j < now; j += blockDim.x >> 5) {
            const uint32_t p = I.select_warp<false>(first + (j - had));
            if ((threadIdx.x & 31) == 0) {
                row[j] = (int32_t)p;
                P.ref[p] = 1;
            }
        }
        return;
    }
    for (uint32_t j = had + threadIdx.x; j < now; j += blockDim.x) {
        const uint32_t p = I.select<false>(first + (j - had));
        row[j] = (int32_t)p;
        P.ref[p] = 1;
    }
}

// blockIdx.x: entry; blockIdx.y == 0 writes its row, and every blockIdx.y copies the tail in its share
// of the layers' keys and values.
__global__ void __launch_bounds__(256) k_pages_fork(const __grid_constant__ pages_in P, const __grid_constant__ pages_scan S,
                                                    uint32_t n)
{
    cr_launch_next();
    cr_wait_previous();
    __shared__ uint32_t pre[kMaxChunks + 1];
    page_index I;
    I.build(S, pre);
    const bool ok = *S.need <= I.free_pages();
    const bool first = blockIdx.y == 0;
    if (!ok && first && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(P.status, CR_FLAG_NOPAGES);
    const int4 e = S.entry[blockIdx.x];
    if (e.x < 0) return;
    if (first && threadIdx.x == 0) P.lens[e.x] = ok ? e.z : 0;
    if (!ok) return;
    const uint32_t full = (uint32_t)e.z >> P.page_log2, tail = (uint32_t)e.z & (P.page - 1);
    const int32_t *src = P.table + (uint64_t)e.y * P.max_pages;
    int32_t *dst = P.table + (uint64_t)e.x * P.max_pages;
    if (first)
        for (uint32_t j = threadIdx.x; j < full; j += blockDim.x) {
            const int p = src[j];
            dst[j] = p;
            if (p >= 0 && (uint32_t)p < P.n_pages)
                atomicAdd(P.ref + p, 1);
            else
                atomicOr(P.status, CR_FLAG_BADPAGES);
        }
    if (!tail) return;
    const uint32_t to = I.select_warp<false>(S.base[blockIdx.x]);
    const int from = src[full];
    if (first && threadIdx.x == 0) {
        dst[full] = (int32_t)to;
        P.ref[to] = 1;
    }
    if (from < 0 || (uint32_t)from >= P.n_pages) {
        if (first && threadIdx.x == 0) atomicOr(P.status, CR_FLAG_BADPAGES);
        return;
    }
    const bool by_token = P.token_stride >= P.head_stride;  // the page's tokens lie one after the other
    const uint32_t segs = by_token ? 1 : P.kv_heads;
    const uint32_t words = (tail * P.head_dim << P.size_log2) / 16 * (by_token ? P.kv_heads : 1);
    // one warp copies a segment, or several where there are fewer segments than warps
    const uint32_t nseg = (2 * P.layers - blockIdx.y + gridDim.y - 1) / gridDim.y * segs, nw = blockDim.x >> 5;
    const uint32_t share = nseg < nw ? nw / nseg : 1, warp = threadIdx.x >> 5;
    for (uint32_t g = warp / share; g < nseg; g += nw / share) {
        uint8_t *base = P.plane(blockIdx.y + g / segs * gridDim.y) + (g % segs * P.head_stride << P.size_log2);
        uint4 *out = reinterpret_cast<uint4 *>(base + (to * P.page_stride << P.size_log2));
        const uint4 *in = reinterpret_cast<const uint4 *>(base + ((uint64_t)from * P.page_stride << P.size_log2));
        const uint32_t step = 32 * share;
        for (uint32_t i = warp % share * 32 + (threadIdx.x & 31); i < words; i += 4 * step) {  // four loads in flight
            uint4 v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e * step < words) v[e] = in[i + e * step];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e * step < words) out[i + e * step] = v[e];
        }
    }
    if (!P.scale) return;  // the blocks that hold the tail, the last of them perhaps in part
    const uint32_t nb = 1u << (P.page_log2 - P.block_log2), used = ((tail - 1) >> P.block_log2) + 1;
    for (uint32_t l2 = blockIdx.y; l2 < 2 * P.layers; l2 += gridDim.y)
        for (uint32_t i = threadIdx.x; i < P.kv_heads * nb; i += blockDim.x)
            if ((i & (nb - 1)) < used) P.scales(l2, to)[i] = P.scales(l2, (uint32_t)from)[i];
}

// A block per entry.
__global__ void __launch_bounds__(128) k_pages_free(const __grid_constant__ pages_in P, const int32_t *seqs)
{
    cr_launch_next();
    cr_wait_previous();
    __shared__ int len;
    const int row = seqs[blockIdx.x];
    if (row < 0 || (uint32_t)row >= P.n_seqs) {
        if (threadIdx.x == 0) atomicOr(P.status, CR_FLAG_BADPAGES);
        return;
    }
    if (threadIdx.x == 0) len = atomicExch(P.lens + row, 0);  // a row that is listed twice is freed once
    __syncthreads();
    int32_t *t = P.table + (uint64_t)row * P.max_pages;
    uint32_t used = len > 0 ? pages_of((uint32_t)len, P.page_log2) : 0;
    if (len < 0 || used > P.max_pages) {
        if (threadIdx.x == 0) atomicOr(P.status, CR_FLAG_BADPAGES);
        used = used > P.max_pages ? P.max_pages : used;
    }
    for (uint32_t j = threadIdx.x; j < used; j += blockDim.x) {
        const int p = t[j];
        t[j] = -1;
        if (p >= 0 && (uint32_t)p < P.n_pages && atomicSub(P.ref + p, 1) > 0) continue;
        if (p >= 0 && (uint32_t)p < P.n_pages) atomicAdd(P.ref + p, 1);
        atomicOr(P.status, CR_FLAG_BADPAGES);
    }
}

// Blocks 0 .. b_pages-1: the new counts and the map; .. b_table-1: tables; the rest: page data.
__global__ void __launch_bounds__(256) k_pages_compact(const __grid_constant__ pages_in P, const __grid_constant__ pages_scan S,
                                                       int32_t *ref_out, int32_t *table_out, int32_t *map, int32_t *live,
                                                       uint32_t b_pages, uint32_t b_table)
{
    cr_launch_next();
    cr_wait_previous();
    __shared__ uint32_t pre[kMaxChunks + 1];
    page_index I;
    I.build(S, pre);
    const uint32_t L = P.n_pages - I.free_pages();
    const uint32_t low = L - I.rank_free(L);  // live pages below L; the others move
    if (blockIdx.x < b_pages) {
        for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < P.n_pages; i += (uint64_t)b_pages * 256) {
            const uint32_t p = (uint32_t)i;
            const bool is_free = (S.bits[p >> 5] >> (p & 31)) & 1;
            int to = -1, ref = 0;
            if (!is_free) to = p < L ? (int)p : (int)I.select<false>(p - I.rank_free(p) - low);
            if (p < L) ref = P.ref[is_free ? I.select<true>(low + I.rank_free(p)) : p];
            map[p] = to;
            ref_out[p] = ref;
        }
        if (blockIdx.x == 0 && threadIdx.x == 0) *live = (int32_t)L;
    } else if (blockIdx.x < b_table) {
        const uint64_t n = (uint64_t)P.n_seqs * P.max_pages;
        const uint64_t step = (uint64_t)(b_table - b_pages) * 256;
        for (uint64_t i = (uint64_t)(blockIdx.x - b_pages) * 256 + threadIdx.x; i < n; i += step) {
            const int p = P.table[i];
            int to = -1;
            if (p >= 0) {
                if ((uint32_t)p >= P.n_pages || ((S.bits[p >> 5] >> (p & 31)) & 1))
                    atomicOr(P.status, CR_FLAG_BADPAGES);
                else
                    to = (uint32_t)p < L ? p : (int)I.select<false>(p - I.rank_free(p) - low);
            }
            table_out[i] = to;
        }
    } else {
        // an equal share of the (move, plane) pairs, in batches whose pages the threads look up together
        __shared__ uint32_t from[256], to[256];
        const uint32_t words = (P.page * P.kv_heads * P.head_dim << P.size_log2) / 16, planes = 2 * P.layers,
                       nb = gridDim.x - b_table;
        const uint64_t n = (uint64_t)(L - low) * planes, b = blockIdx.x - b_table;
        for (uint64_t i = n * b / nb, end = n * (b + 1) / nb; i < end;) {
            const uint32_t k0 = (uint32_t)(i / planes), k = k0 + threadIdx.x;
            const uint64_t stop = min(end, ((uint64_t)k0 + 256) * planes);
            __syncthreads();
            if ((uint64_t)k * planes < stop) {
                from[threadIdx.x] = I.select<true>(low + k);
                to[threadIdx.x] = I.select<false>(k);
            }
            __syncthreads();
            for (; i < stop; ++i) {
                const uint32_t m = (uint32_t)(i / planes) - k0;
                const uint32_t l2 = (uint32_t)(i % planes);
                uint8_t *base = P.plane(l2);
                copy16(reinterpret_cast<uint4 *>(base + (to[m] * P.page_stride << P.size_log2)),
                       reinterpret_cast<const uint4 *>(base + (from[m] * P.page_stride << P.size_log2)), words);
                if (P.scale)
                    for (uint32_t j = threadIdx.x; j < P.kv_heads << (P.page_log2 - P.block_log2); j += blockDim.x)
                        P.scales(l2, to[m])[j] = P.scales(l2, from[m])[j];
            }
        }
    }
}

struct write_in {
    const uint16_t *k, *v;
    uint64_t k_token, k_head, v_token, v_head;
    const int32_t *cu, *seqs;
    uint32_t n, n_tokens, wpt_log2;
};

// 2^wpt_log2 warps per token; 16 bytes a lane.
__global__ void __launch_bounds__(128) k_kv_write(const __grid_constant__ pages_in P, const __grid_constant__ write_in W,
                                                  uint32_t layer)
{
    cr_launch_next();
    cr_wait_previous();
    const uint64_t warp = ((uint64_t)blockIdx.x * 128 + threadIdx.x) >> 5;
    const uint64_t t = warp >> W.wpt_log2;
    if (t >= W.n_tokens) return;
    // entry: the last whose tokens begin at or before t, 32 looks at a time
    const uint32_t lane = threadIdx.x & 31;
    uint32_t lo = 0, span = W.n + 1;
    while (span > 1) {
        const uint32_t step = (span + 31) / 32, i = lo + lane * step;
        const bool in = lane * step < span && W.cu[i] <= (int)t;
        const uint32_t some = __ballot_sync(~0u, in), last = some ? 31 - __clz(some) : 0;
        lo += last * step;
        span = min(step, span - last * step);
    }
    bool ok = lo < W.n && W.cu[lo] <= (int)t && (int)t < W.cu[lo + 1];
    ++lo;
    uint64_t dst = 0;
    if (ok) {
        const int row = W.seqs ? W.seqs[lo - 1] : (int)lo - 1;
        ok = row >= 0 && (uint32_t)row < P.n_seqs;
        if (ok) {
            const int pos = P.lens[row] - (W.cu[lo] - (int)t);
            ok = pos >= 0 && ((uint32_t)pos >> P.page_log2) < P.max_pages;
            if (ok) {
                const int p = P.table[(uint64_t)row * P.max_pages + ((uint32_t)pos >> P.page_log2)];
                // pages that other rows name are not this row's to write: a row that was not grown (too wide, too few
                // pages) would put its tokens there
                ok = p >= 0 && (uint32_t)p < P.n_pages && P.ref[p] <= 1;
                dst = (uint64_t)(uint32_t)p * P.page_stride + ((uint32_t)pos & (P.page - 1)) * P.token_stride;
            }
        }
    }
    if (!ok) {
        if ((threadIdx.x & 31) == 0) atomicOr(P.status, CR_FLAG_BADPAGES);
        return;
    }
    const uint32_t per = P.head_dim / 8, words = P.kv_heads * per, step = 32u << W.wpt_log2;
    uint16_t *kd = reinterpret_cast<uint16_t *>(P.plane(2 * layer)) + dst;
    uint16_t *vd = reinterpret_cast<uint16_t *>(P.plane(2 * layer + 1)) + dst;
    const uint16_t *ks = W.k + t * W.k_token, *vs = W.v + t * W.v_token;
    for (uint32_t i = (threadIdx.x & 31) + 32 * (uint32_t)(warp & ((1u << W.wpt_log2) - 1)); i < words; i += step) {
        const uint32_t h = i / per, d = (i - h * per) * 8;
        const uint4 a = *reinterpret_cast<const uint4 *>(ks + h * W.k_head + d);
        const uint4 b = *reinterpret_cast<const uint4 *>(vs + h * W.v_head + d);
        *reinterpret_cast<uint4 *>(kd + h * P.head_stride + d) = a;
        *reinterpret_cast<uint4 *>(vd + h * P.head_stride + d) = b;
    }
}

int scan_mem(cr_ctx *ctx, const cr_kv_pages *pg, uint32_t n, pages_scan &S)
{
    S = pages_scan{};
    S.n_pages = pg->n_pages;
    S.chunk_log2 = 10;
    while ((((uint64_t)pg->n_pages + (1ull << S.chunk_log2) - 1) >> S.chunk_log2) > kMaxChunks) ++S.chunk_log2;
    S.chunks = (uint32_t)(((uint64_t)pg->n_pages + (1ull << S.chunk_log2) - 1) >> S.chunk_log2);
    const size_t words = (size_t)S.chunks << (S.chunk_log2 - 5);
    void *p;
    CR_TRY(cr_scratch(ctx, SCR_PAGES, 16 * ((size_t)n + 1) + 4 * ((size_t)n + 1) + 8 * words + 4 * (size_t)S.chunks + 64, &p));
    S.need = static_cast<unsigned long long *>(p);
    S.entry = reinterpret_cast<int4 *>(static_cast<char *>(p) + 16);
    S.base = reinterpret_cast<uint32_t *>(S.entry + n);
    S.bits = S.base + n;
    S.wpre = S.bits + words;
    S.cnt = S.wpre + words;
    return CR_OK;
}

}  // namespace

int cr_pages_check(cr_ctx *ctx, const char *who, const cr_kv_pages *pg)
{
    if (!pg) return cr_fail(ctx, CR_EINVAL, "%s: pages is NULL", who);
    if (!pg->d_cache || !pg->d_ref || !pg->d_table || !pg->d_lens) return cr_fail(ctx, CR_EINVAL, "%s: NULL pointer in pages", who);
    if (pg->dtype > CR_DTYPE_FP16_E4M3) return cr_fail(ctx, CR_EINVAL, "%s: dtype %u", who, pg->dtype);
    if (pg->page < 8 || pg->page > 256 || (pg->page & (pg->page - 1)))
        return cr_fail(ctx, CR_EINVAL, "%s: page of %u tokens: a power of two, 8..256", who, pg->page);
    if (pg->head_dim == 0 || pg->head_dim > 128 || (pg->head_dim & 7))
        return cr_fail(ctx, CR_EINVAL, "%s: head_dim %u: a multiple of 8, 8..128", who, pg->head_dim);
    if (!pg->layers || pg->layers > 4096 || !pg->kv_heads || pg->kv_heads > 4096 || !pg->n_pages || !pg->n_seqs || !pg->max_pages)
        return cr_fail(ctx, CR_EINVAL, "%s: empty pool (layers, heads, pages, sequences, pages per row)", who);
    if ((uint64_t)pg->n_pages * pg->page >= (1ull << 31) || (uint64_t)pg->max_pages * pg->page >= (1ull << 31) ||
        (uint64_t)pg->n_seqs * pg->max_pages >= (1ull << 40) || pg->n_seqs >= (1u << 31))
        return cr_fail(ctx, CR_EINVAL, "%s: pool too large", who);
    const uint64_t hd = pg->head_dim, row = hd * pg->kv_heads;
    const bool by_token = pg->token_stride == row && pg->head_stride == hd;
    const bool by_head = pg->head_stride == pg->page * hd && pg->token_stride == hd;
    if (!(by_token || by_head) || pg->page_stride < pg->page * row)
        return cr_fail(ctx, CR_EINVAL, "%s: a page's tokens and heads must be dense, one page after the other", who);
    if (((uintptr_t)pg->d_cache & 15) || ((pg->layer_stride | pg->kv_stride | pg->page_stride) & 7))
        return cr_fail(ctx, CR_EINVAL, "%s: the cache must be 16-byte aligned, its strides multiples of 8", who);
    if (pg->page_stride >= (1ull << 38))
        return cr_fail(ctx, CR_EINVAL, "%s: page stride too large", who);
    if (cr_in_8bit(pg->dtype)) {
        if (!pg->d_scale || ((uintptr_t)pg->d_scale & 3)) return cr_fail(ctx, CR_EINVAL, "%s: d_scale must hold the blocks' scales", who);
        if (pg->head_dim & 15) return cr_fail(ctx, CR_EINVAL, "%s: head_dim %u: a multiple of 16 in 8 bits", who, pg->head_dim);
        if (pg->block < 8 || pg->block > pg->page || (pg->block & (pg->block - 1)))
            return cr_fail(ctx, CR_EINVAL, "%s: blocks of %u tokens: a power of two, 8..page", who, pg->block);
        if ((pg->layer_stride | pg->kv_stride | pg->page_stride) & 15)
            return cr_fail(ctx, CR_EINVAL, "%s: strides of a cache in 8 bits must be multiples of 16", who);
        if (pg->reserved) return cr_fail(ctx, CR_EINVAL, "%s: reserved must be 0", who);
    }
    return CR_OK;
}

static int list_check(cr_ctx *ctx, const char *who, uint32_t n, const void *a, const void *b, const void *c)
{
    if (n >= (1u << 24)) return cr_fail(ctx, CR_EINVAL, "%s: %u entries", who, n);
    if (n && (!a || !b || !c)) return cr_fail(ctx, CR_EINVAL, "%s: NULL list", who);
    return CR_OK;
}

extern "C" int cr_pages_extend(cr_ctx *ctx, const cr_kv_pages *pages, const int32_t *d_seqs, const int32_t *d_add, uint32_t n)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_pages_extend");
    CR_TRY(cr_pages_check(ctx, "cr_pages_extend", pages));
    CR_TRY(list_check(ctx, "cr_pages_extend", n, d_seqs, d_add, d_add));
    if (!n) return CR_OK;
    const pages_in P = cr_pages_input(ctx, pages);
    pages_scan S;
    CR_TRY(scan_mem(ctx, pages, n, S));
    CR_TRY(cr_launch_early(ctx, "k_pages_scan", k_pages_scan<SCAN_EXTEND>, dim3(S.chunks + 1), 1024, 0, P, S, d_seqs, d_add, d_add, n));
    CR_TRY(cr_launch_early(ctx, "k_pages_extend", k_pages_extend, dim3(n), 128, 0, P, S, n));
    return CR_OK;
}

extern "C" int cr_pages_fork(cr_ctx *ctx, const cr_kv_pages *pages, const int32_t *d_src, const int32_t *d_dst,
                             const int32_t *d_keep, uint32_t n)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_pages_fork");
    CR_TRY(cr_pages_check(ctx, "cr_pages_fork", pages));
    CR_TRY(list_check(ctx, "cr_pages_fork", n, d_src, d_dst, d_keep));
    if (!n) return CR_OK;
    const pages_in P = cr_pages_input(ctx, pages);
    pages_scan S;
    CR_TRY(scan_mem(ctx, pages, n, S));
    CR_TRY(cr_launch_early(ctx, "k_pages_scan", k_pages_scan<SCAN_FORK>, dim3(S.chunks + 1), 1024, 0, P, S, d_src, d_dst, d_keep, n));
    // few entries: several blocks copy the layers of each (8 are resident on every SM)
    uint32_t fork_split = 8 * (uint32_t)ctx->num_sms / n;
    fork_split = fork_split < 1 ? 1 : (fork_split > 2 * pages->layers ? 2 * pages->layers : fork_split);
    CR_TRY(cr_launch_early(ctx, "k_pages_fork", k_pages_fork, dim3(n, fork_split), 256, 0, P, S, n));
    return CR_OK;
}

extern "C" int cr_pages_free(cr_ctx *ctx, const cr_kv_pages *pages, const int32_t *d_seqs, uint32_t n)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_pages_free");
    CR_TRY(cr_pages_check(ctx, "cr_pages_free", pages));
    CR_TRY(list_check(ctx, "cr_pages_free", n, d_seqs, d_seqs, d_seqs));
    if (!n) return CR_OK;
    const pages_in P = cr_pages_input(ctx, pages);
    CR_TRY(cr_launch_early(ctx, "k_pages_free", k_pages_free, dim3(n), 128, 0, P, d_seqs));
    return CR_OK;
}

extern "C" int cr_pages_compact(cr_ctx *ctx, const cr_kv_pages *pages, int32_t *d_ref_out, int32_t *d_table_out, int32_t *d_map,
                                int32_t *d_live)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_pages_compact");
    CR_TRY(cr_pages_check(ctx, "cr_pages_compact", pages));
    if (!d_ref_out || !d_table_out || !d_map || !d_live) return cr_fail(ctx, CR_EINVAL, "cr_pages_compact: NULL output");
    if (d_ref_out == pages->d_ref || d_table_out == pages->d_table)
        return cr_fail(ctx, CR_EINVAL, "cr_pages_compact: the outputs must be arrays of their own");
    const pages_in P = cr_pages_input(ctx, pages);
    pages_scan S;
    CR_TRY(scan_mem(ctx, pages, 0, S));
    const int32_t *none = nullptr;
    CR_TRY(cr_launch_early(ctx, "k_pages_scan", k_pages_scan<SCAN_NONE>, dim3(S.chunks), 1024, 0, P, S, none, none, none, 0u));
    const uint32_t sms = (uint32_t)ctx->num_sms;
    const uint32_t b_pages = cr_blocks(pages->n_pages, 256, 2 * sms);
    const uint32_t b_table = b_pages + cr_blocks((uint64_t)pages->n_seqs * pages->max_pages, 1024, 2 * sms);
    CR_TRY(cr_launch_early(ctx, "k_pages_compact", k_pages_compact, dim3(b_table + 8 * sms), 256, 0, P, S, d_ref_out, d_table_out, d_map, d_live, b_pages, b_table));
    return CR_OK;
}

extern "C" int cr_kv_write(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, const void *d_k, uint64_t k_token,
                           uint64_t k_head, const void *d_v, uint64_t v_token, uint64_t v_head, const int32_t *d_cu,
                           const int32_t *d_seqs, uint32_t n, uint32_t n_tokens)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_kv_write");
    CR_TRY(cr_pages_check(ctx, "cr_kv_write", pages));
    if (layer >= pages->layers) return cr_fail(ctx, CR_EINVAL, "cr_kv_write: layer %u of %u", layer, pages->layers);
    if (n > (1u << 24) || n_tokens > (1u << 30)) return cr_fail(ctx, CR_EINVAL, "cr_kv_write: too many entries or tokens");
    if (!n || !n_tokens) return CR_OK;
    if (!d_k || !d_v || !d_cu) return cr_fail(ctx, CR_EINVAL, "cr_kv_write: NULL pointer");
    if (((uintptr_t)d_k & 15) || ((uintptr_t)d_v & 15) || ((k_token | k_head | v_token | v_head) & 7))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_write: keys and values must be 16-byte aligned, strides multiples of 8");
    if (cr_in_8bit(pages->dtype)) {
        cr_append_args A = {};
        A.d_k = d_k;
        A.d_v = d_v;
        A.k_token = k_token;
        A.k_head = k_head;
        A.v_token = v_token;
        A.v_head = v_head;
        A.d_cu = d_cu;
        A.d_seqs = d_seqs;
        A.n = n;
        A.n_tokens = n_tokens;
        return cr_append(ctx, "cr_kv_write", pages, layer, nullptr, &A);
    }
    const pages_in P = cr_pages_input(ctx, pages);
    write_in W = {static_cast<const uint16_t *>(d_k), static_cast<const uint16_t *>(d_v), k_token, k_head, v_token, v_head,
                  d_cu, d_seqs, n, n_tokens, 0};
    // few tokens: more warps on each, as long as they have words to move
    while (W.wpt_log2 < 3 && ((uint64_t)n_tokens << W.wpt_log2) < 8ull * ctx->num_sms &&
           (32u << W.wpt_log2) < pages->kv_heads * (pages->head_dim / 8))
        ++W.wpt_log2;
    const uint64_t warps = (uint64_t)n_tokens << W.wpt_log2;
    CR_TRY(cr_launch_early(ctx, "k_kv_write", k_kv_write, dim3((uint32_t)((warps + 3) / 4)), 128, 0, P, W, layer));
    return CR_OK;
}
