// Attention over packed prompts, over cached pages, and of single tokens that share a prefix
// (include/cacheroute.h).
//
// Every call is one softmax over the keys a query sees, taken a tile of keys at a time with the
// running maximum m and sum l of its row (o, l scaled by 2^(m_old - m_new) when m grows), so a
// row's result is (m, l, o) of any subset of its keys, and two of them join exactly:
//   m = max(m1, m2),  l = l1 2^(m1-m) + l2 2^(m2-m),  o = o1 2^(m1-m) + o2 2^(m2-m).
// Work is therefore a list of (key head, block of query rows) with a number of key tiles each,
// laid end to end; every CTA takes an equal stretch of it, wherever that begins or ends.  What a
// CTA has of a block that it shares with others goes to scratch, and a second kernel joins the
// pieces in order (k_attn_plan, one CTA, writes the list and the stretches, but for a few single tokens,
// whose list k_attn_few makes).  A block counts for its tiles and for some more
// (extra): its queries, its first scores and its result, which no other work hides.
//
// Two kernels do the work:
//   k_attn_rows  many query rows per key head: 256 rows (tokens x grouped heads) against tiles of
//                128 keys on the tensor cores with accumulators in tensor memory;
//   k_attn_few   at most 16 rows per key head (one token's grouped heads): tiles of 64 keys.
#include <math.h>

#include "cr_attn_index.cuh"
#include "cr_pages.cuh"
#include "cr_tensor.cuh"

namespace {

constexpr int kRowsTile = 128;  // query rows of a tile, and keys of one
constexpr int kFewTile = 64;    // keys of a tile of k_attn_few
constexpr int kFewWarps = 4;
constexpr uint32_t kExtra = 1;
// Weights are exp2 of one fused operation, score * c - maximum * c, whose second product is a rounded one.  Where that is
// beyond this size (a base-2 logarithm) what the rounding drops is no longer small in an exponent, and even the largest
// weight could overflow or vanish.  There c becomes its power of two, with which both products are exact: distinct scores
// are still 2^-3 or more apart, and have 32-bit sums' errors of 2^4 at least.
constexpr float kFar = 0x1p22f;
inline float coarse(float c) { return fmaxf(ldexpf(0.5f, ilogbf(c) + 1), 0x1p-126f); }
// Single tokens over 8 bits: a tile takes half of the time, and a block's beginning and end the same.
constexpr uint32_t kFewExtra8 = 4;

// A block of query rows of one key head.
struct __align__(16) attn_blk {
    int row0;   // its first query token
    int ntok;   // its query tokens
    int klen;   // keys of its sequence
    int kbase;  // packed: first key token; paged: row of the table
    int diag;   // keys before the one that its first query token sees last (causal)
    int lo;     // k_attn_few: keys below are already counted (the shared prefix)
    int nt;     // its key tiles
    int pad;
};
// Where a CTA's stretch begins.
struct __align__(16) attn_start {
    unsigned long long pos, N;  // N: key tiles of all stretches
    uint32_t head, blk, tile, nblk;
    attn_blk k;                 // its first block
    // where the stretch is the first to begin inside that block: the block's pieces (from the stretch before on)
    uint32_t pieces, pad[3];
};
constexpr uint32_t kMaxCtas = 511;

// What the plan kernel reads.
struct plan_in {
    const int32_t *cu_q;   // NULL: one token per entry
    const int32_t *cu_k;   // packed
    const int32_t *seqs;   // paged: row of each entry (NULL: i)
    const int32_t *lens;   // paged
    const int32_t *goff, *shared;  // groups
    uint32_t n, n_tokens, n_kv, n_seqs, n_groups, heads, max_blk, max_cta, causal;
    uint32_t tok_blk;      // query tokens per block
    uint32_t max_len;      // paged: tokens that a row can hold
    uint32_t min_tiles;    // key tiles that a CTA is worth
    uint32_t piece_cost;   // what a piece costs, in key tiles
    uint32_t extra;        // what a block does
    attn_blk *blk;
    attn_start *start;        // [max_cta + 1]
    uint32_t *joins;          // [max_cta + 1] number of blocks with several pieces, and their first stretches
    // of long lists only (the plan kernel's shared memory holds the others)
    unsigned long long *cum;  // [max_blk + 1] key tiles before each block
    uint32_t *first;          // [n + 1] first block of each entry
    int32_t *of_token;        // groups: first token of each query token's block
};
constexpr uint32_t kPlanShared = 512;
struct plan_shared {
    unsigned long long cum[kPlanShared + 1], pos[kMaxCtas + 1];
    unsigned long long end[kMaxCtas + 1];  // of the block that a stretch begins inside, or 0
    unsigned long long part[32];
    uint32_t first_tile[kMaxCtas + 1];
    uint32_t first[kPlanShared + 1], joins, longest;
    int goff[kPlanShared + 1], keys[kPlanShared];  // groups
    attn_blk blk[kPlanShared];
};

enum { PLAN_PACKED, PLAN_PAGED, PLAN_GROUPS, PLAN_FEW };

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// Exclusive scan over the CTA's NT threads; *total receives the sum.
template <int NT>
__device__ unsigned long long scan_cta(unsigned long long v, unsigned long long *part, unsigned long long *total)
{
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    unsigned long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(~0u, x, o);
        if (lane >= (uint32_t)o) x += y;
    }
    if (lane == 31) part[w] = x;
    __syncthreads();
    unsigned long long before = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) {
        const unsigned long long y = part[i];
        if (i < (int)w) before += y;
        sum += y;
    }
    *total = sum;
    __syncthreads();
    return before + x - v;
}

__device__ __forceinline__ void q_range(const plan_in &A, uint32_t i, int &lo, int &hi)
{
    if (!A.cu_q) {
        lo = (int)i;
        hi = (int)i + 1;
        return;
    }
    lo = clampi(A.cu_q[i], 0, (int)A.n_tokens);
    hi = clampi(A.cu_q[i + 1], lo, (int)A.n_tokens);
}

// Row of the table of an entry, or -1; its keys.
__device__ __forceinline__ int row_of(const plan_in &A, int e)
{
    const int row = A.seqs ? A.seqs[e] : e;
    return row >= 0 && (uint32_t)row < A.n_seqs ? row : -1;
}
__device__ __forceinline__ int keys_of(const plan_in &A, int row)
{
    return row < 0 ? 0 : clampi(A.lens[row], 0, (int)A.max_len);
}
// Keys that a group's members share, where it has several: they are read once for all.  The first member's length
// bounds them.
__device__ __forceinline__ int group_keys(const plan_in &A, uint32_t g)
{
    const int lo = A.goff[g], hi = A.goff[g + 1];
    const int keys = clampi(A.shared[g], 0, (int)A.max_len);
    if (lo < 0 || lo >= (int)A.n) return 0;
    const int have = keys_of(A, row_of(A, lo));
    return hi - lo < 2 ? 0 : (keys < have ? keys : have);
}

// Last index of a[0 .. n] (ascending) at or below v; a[0] is.
template <typename T>
__device__ __forceinline__ uint32_t at_or_below(const T *a, uint32_t n, T v)
{
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t m = (lo + hi + 1) >> 1;
        if (a[m] <= v)
            lo = m;
        else
            hi = m - 1;
    }
    return lo;
}

// One CTA makes a list; what it takes (about 6,000 cycles for a few blocks) is reads, barriers and searches one
// after the other, so attention kernels begin their own prologues meanwhile.
// Most lists are short: their divisions are done in 32 bits.
__device__ __forceinline__ unsigned long long div_by(unsigned long long a, unsigned long long b)
{
    return a >> 32 || b >> 32 ? a / b : (uint32_t)a / (uint32_t)b;
}

// How the work is cut: N units in stretches of equal length, or one stretch for each block.
struct plan_cut {
    unsigned long long N, Nb, snap;
    uint32_t nblk, ncta, extra;
    bool one_each;
};
// Nb: of a head; filled: blocks that have keys; longest: their most tiles.
__device__ __forceinline__ plan_cut cut_work(const plan_in &A, unsigned long long Nb, uint32_t nblk, uint32_t filled,
                                             uint32_t longest)
{
    plan_cut C;
    C.extra = A.extra;
    C.Nb = Nb;
    C.nblk = nblk;
    C.N = Nb * A.heads;  // N < 2^54
    const unsigned long long want = div_by(C.N, A.min_tiles);
    C.ncta = want < 1 ? 1u : (want < A.max_cta ? (uint32_t)want : A.max_cta);
    // Few blocks.  One stretch for each block leaves no pieces; where that is too long, as many for each, so that most
    // stretches are within one block and leave one piece instead of two.  Both where they make the longest stretch
    // longer by less than a piece costs (its result's way to scratch and back).
    const unsigned long long blocks = (unsigned long long)filled * A.heads;
    C.one_each = false;
    if (blocks && blocks <= A.max_cta) {
        const unsigned long long most_now = div_by(C.N, C.ncta) + A.piece_cost;
        if (filled == nblk && longest + A.extra <= most_now) {
            C.one_each = true;
            C.ncta = (uint32_t)blocks;
        } else if (blocks <= C.ncta) {
            const uint32_t even = C.ncta / (uint32_t)blocks * (uint32_t)blocks;
            if (div_by(C.N, even) <= most_now) C.ncta = even;
        }
    }
    C.snap = div_by(C.N, C.ncta) / 8;  // a stretch ends with its block where that is near
    return C;
}

// Where stretch c begins; cum: units before each block.
__device__ __forceinline__ attn_start stretch(const plan_cut &C, const unsigned long long *cum, const attn_blk *blk,
                                              uint32_t c)
{
    attn_start s = {};
    s.pos = c < C.ncta ? div_by(C.N * c, C.ncta) : C.N;
    if (C.one_each && c < C.ncta) {
        s.head = c / C.nblk;
        s.blk = c - s.head * C.nblk;
        s.pos = s.head * C.Nb + cum[s.blk];
    } else if (s.pos < C.N) {
        s.head = (uint32_t)div_by(s.pos, C.Nb);
        const unsigned long long rem = s.pos - s.head * C.Nb;
        s.blk = at_or_below(cum, C.nblk, rem);
        const unsigned long long t = rem - cum[s.blk], left = cum[s.blk + 1] - rem;
        s.tile = (uint32_t)(t - C.extra);
        if (t <= C.snap || t <= C.extra) {
            s.pos -= t;
            s.tile = 0;
        } else if (left <= C.snap) {
            s.pos += left;
            s.tile = 0;
            if (++s.blk == C.nblk) {
                s.blk = 0;
                ++s.head;
            }
        }
    }
    s.N = C.N;
    s.nblk = C.nblk;
    if (s.pos < C.N) {
        while (cum[s.blk + 1] == cum[s.blk])  // blocks without keys
            if (++s.blk == C.nblk) {
                s.blk = 0;
                ++s.head;
            }
        s.k = blk[s.blk];
    }
    return s;
}

template <int KIND, int NT>
__device__ void plan_build(const plan_in &A, plan_shared &S, uint32_t *status)
{
    const uint32_t tid = threadIdx.x;
    const uint32_t n = KIND == PLAN_GROUPS ? A.n_groups : A.n;
    uint32_t *first = n <= kPlanShared ? S.first : A.first;
    const bool near = A.max_blk <= kPlanShared;
    unsigned long long *cum = near ? S.cum : A.cum;
    unsigned long long total, base = 0;
    if (tid == 0) S.joins = S.longest = 0;
    // blocks of every entry
    uint32_t nblk = n;
    if (KIND != PLAN_FEW) {
        for (uint32_t i0 = 0; i0 < n; i0 += NT) {
            const uint32_t i = i0 + tid;
            unsigned long long nb = 0;
            if (i < n) {
                int lo, hi;
                q_range(A, i, lo, hi);
                nb = ((uint32_t)(hi - lo) + A.tok_blk - 1) / A.tok_blk;
            }
            const unsigned long long at = base + scan_cta<NT>(nb, S.part, &total);
            if (i < n) first[i] = (uint32_t)(at < A.max_blk ? at : A.max_blk);
            base += total;
        }
        if (base > A.max_blk) {  // entries that overlap: not ascending
            if (tid == 0) atomicOr(status, CR_FLAG_BADPAGES);
            base = A.max_blk;
        }
        nblk = (uint32_t)base;
        if (tid == 0) first[n] = nblk;
        __syncthreads();
    } else if (A.n_groups && A.n_groups <= kPlanShared) {
        for (uint32_t g = tid; g < A.n_groups; g += NT) {
            S.keys[g] = group_keys(A, g);
            S.goff[g] = A.goff[g];
            if (A.goff[g] > A.goff[g + 1]) atomicOr(status, CR_FLAG_BADPAGES);
        }
        if (tid == 0) S.goff[A.n_groups] = A.goff[A.n_groups];
        __syncthreads();
    }
    // their keys
    uint32_t filled = 0;  // blocks that have any
    unsigned long long most = 0;
    base = 0;
    for (uint32_t b0 = 0; b0 < nblk; b0 += NT) {
        const uint32_t b = b0 + tid;
        unsigned long long nt = 0;
        attn_blk k = {};
        if (b < nblk) {
            const uint32_t i = KIND == PLAN_FEW ? b : at_or_below(first, n, b);
            int lo, hi;
            q_range(A, i, lo, hi);
            k.row0 = lo;
            k.ntok = hi - lo;
            if (KIND != PLAN_FEW) {
                const int t0 = (int)((b - first[i]) * A.tok_blk);
                k.row0 = lo + t0;
                k.ntok = clampi(hi - lo - t0, 0, (int)A.tok_blk);
            }
            if (KIND == PLAN_PACKED) {
                const int klo = clampi(A.cu_k[i], 0, (int)A.n_kv), khi = clampi(A.cu_k[i + 1], klo, (int)A.n_kv);
                k.kbase = klo;
                k.klen = khi - klo;
            } else {
                const int e = KIND == PLAN_GROUPS ? lo : (int)i;  // entry whose row is read
                const int row = e < (int)A.n ? row_of(A, e) : -1;
                if (row < 0 && e < (int)A.n) atomicOr(status, CR_FLAG_BADPAGES);
                k.kbase = row < 0 ? 0 : row;
                k.klen = KIND == PLAN_GROUPS ? group_keys(A, i) : keys_of(A, row);
                if (KIND == PLAN_FEW && A.n_groups) {
                    const bool in_shared = A.n_groups <= kPlanShared;
                    const int *goff = in_shared ? S.goff : A.goff;
                    if (goff[0] <= (int)i) {
                        const uint32_t g = at_or_below(goff, A.n_groups, (int)i);
                        if (g < A.n_groups) k.lo = in_shared ? S.keys[g] : group_keys(A, g);
                        if (k.lo > k.klen) atomicOr(status, CR_FLAG_BADPAGES);
                    }
                }
            }
            int end = k.klen;
            if (KIND == PLAN_PACKED || KIND == PLAN_PAGED) {
                k.diag = k.klen - (hi - lo) + (k.row0 - lo);
                if (A.causal) end = clampi(k.diag + k.ntok, 0, k.klen);
            }
            if (KIND == PLAN_FEW) {
                nt = cr_few_tiles(k.lo, k.klen, kFewTile);
            } else {
                nt = cr_key_tiles(end, kRowsTile);
                if (nt == 0 && KIND != PLAN_GROUPS) nt = 1;  // rows without keys: zeros
            }
            k.nt = (int)nt;
            if (KIND == PLAN_GROUPS)
                for (int t = 0; t < k.ntok; ++t) A.of_token[k.row0 + t] = k.row0;
        }
        filled += __syncthreads_count(nt > 0);
        const unsigned long long at = base + scan_cta<NT>(nt ? nt + A.extra : 0, S.part, &total);
        if (b < nblk) {
            cum[b] = at;
            A.blk[b] = k;
            if (near) S.blk[b] = k;
            if (nt > most) most = nt;
        }
        base += total;
    }
    if (tid == 0) cum[nblk] = base;
    if (most) atomicMax(&S.longest, (uint32_t)most);
    __syncthreads();
    // stretches
    const plan_cut C = cut_work(A, base, nblk, filled, S.longest);
    for (uint32_t c = tid; c <= A.max_cta; c += NT) {
        const attn_start s = stretch(C, cum, near ? S.blk : A.blk, c);
        A.start[c] = s;
        S.pos[c] = s.pos;
        S.end[c] = s.tile && s.pos < C.N ? s.pos - s.tile + (uint32_t)s.k.nt : 0;
        S.first_tile[c] = s.tile;
    }
    __syncthreads();
    // the first stretch that begins inside a block joins its pieces
    for (uint32_t c = 1 + tid; c < C.ncta; c += NT) {
        if (S.end[c] == 0 || S.pos[c - 1] > S.pos[c] - S.first_tile[c] - A.extra) continue;
        A.start[c].pieces = at_or_below(S.pos, A.max_cta, S.end[c] - 1) + 1 - (c - 1);
        A.joins[1 + atomicAdd(&S.joins, 1)] = c;  // in any order
    }
    __syncthreads();
    if (tid == 0) A.joins[0] = S.joins;
}

template <int KIND, int NT>
__global__ void __launch_bounds__(NT) k_attn_plan(const __grid_constant__ plan_in a, const __grid_constant__ plan_in b,
                                                  uint32_t *status)
{
    __shared__ plan_shared S;
    cr_launch_next();
    cr_wait_previous();
    if (blockIdx.x == 0)
        plan_build<KIND, NT>(a, S, status);
    else
        plan_build<PLAN_GROUPS, NT>(b, S, status);
}

// What the attention kernels read.
struct attn_in {
    const attn_blk *blk;
    const attn_start *start;
    const uint32_t *joins;
    int32_t *first_cta, *last_cta;  // single tokens: CTAs that begin and end each (block, head)
    const int32_t *table;  // paged
    uint32_t max_pages, page_log2, box_rows, box_log2;
    uint32_t paged, causal, G, nsub, tq, q_heads, head_dim;
    float c;               // scale * log2(e)
    float c_pow, c_rest;   // its power of two, which stands for it beyond kFar, and what that leaves
    float far;             // kFar / c
    void *o;
    float *lse;
    uint64_t o_token, o_head;
    float *part, *part_ml; // pieces
    float *pfx, *pfx_lse;  // shared prefix: o and log2 of the sum, [token][head]
    float *own, *own_ml;   // k_attn_few: whole blocks that a shared prefix still joins
    const int32_t *of_token;  // groups: first token of each query token's block
    uint32_t kv_heads, few_heads, after_rows, ncta;
    uint32_t to_pfx;       // k_attn_rows, its join: write those instead of o
    uint32_t o_wide;       // rows of o begin at multiples of 32 bytes
    uint32_t *status;
    uint32_t extra;        // of a block, in the list of work
    uint32_t own_list;     // k_attn_few, its join: every CTA makes the list of work itself, from
    plan_in plan;
    // keys and values in 8 bits: their blocks' scales in this layer, [n_pages][kv_heads][1 << nb_log2]
    const float *k_scale, *v_scale;
    uint32_t block_log2, nb_log2, n_pages;
};

// A short list of single tokens: a warp makes it in every CTA, a token a lane, which saves the plan kernel's launch and
// its run before this one's (32/8 heads of 128, calls back to back: one sequence of 2,048 keys 15.0 us with that kernel
// and 12.6 so, eight 20.9 and 18.3, 32 65.3 and 61.8).
constexpr uint32_t kOwnList = 32;
struct own_list {
    attn_start start[2];        // this CTA's stretch and the next
    unsigned long long before;  // where the one before begins
    attn_blk blk[kOwnList];
    unsigned long long cum[kOwnList + 1];
};
__device__ __forceinline__ plan_cut make_list(const plan_in &P, own_list *L, uint32_t *status)
{
    const uint32_t lane = threadIdx.x & 31;
    attn_blk k = {};
    unsigned long long at = 0;
    if (lane < P.n) {
        const int row = row_of(P, (int)lane);
        if (row < 0 && blockIdx.x == 0) atomicOr(status, CR_FLAG_BADPAGES);
        k.row0 = (int)lane;
        k.ntok = 1;
        k.kbase = row < 0 ? 0 : row;
        k.klen = keys_of(P, row);
        k.nt = (int)cr_few_tiles(0, k.klen, kFewTile);
        at = (uint32_t)k.nt + P.extra;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(~0u, at, o);
        if ((int)lane >= o) at += y;
    }
    L->blk[lane] = k;
    L->cum[lane + 1] = at;
    if (lane == 0) L->cum[0] = 0;
    __syncwarp();
    const plan_cut C = cut_work(P, L->cum[P.n], P.n, P.n, __reduce_max_sync(~0u, (uint32_t)k.nt));
    if (lane < 3) {
        const uint32_t c = blockIdx.x + lane - 1;  // the stretch before, this one, the next
        const attn_start s = stretch(C, L->cum, L->blk, c == ~0u ? 0 : c);
        if (lane == 0)
            L->before = s.pos;
        else
            L->start[lane - 1] = s;
        if (lane == 1) P.start[c] = s;
    }
    __syncwarp();
    return C;
}
// Once the copies are under way: if this stretch is the first to begin inside its block, the block's pieces.
__device__ __forceinline__ void count_pieces(const plan_in &P, const plan_cut &C, const own_list *L)
{
    const attn_start &s = L->start[0];
    if (s.tile == 0 || s.pos >= C.N || L->before > s.pos - s.tile - P.extra) return;
    const unsigned long long end = s.pos - s.tile + (uint32_t)s.k.nt;
    // stretches that begin before the block's end: none of them begins a whole stretch from its even share
    const uint32_t near = (uint32_t)div_by(end * C.ncta, C.N), c0 = near > 8 ? near - 8 : 0, c = c0 + (threadIdx.x & 31);
    const uint32_t upto = c0 + __popc(__ballot_sync(~0u, c < C.ncta && stretch(C, L->cum, L->blk, c).pos < end));
    if ((threadIdx.x & 31) == 0) P.start[blockIdx.x].pieces = upto - (blockIdx.x - 1);
}

// A CTA's stretch, a block at a time; the next block's description is on its way while one is worked on.
struct walk {
    unsigned long long left;
    uint32_t extra, h, next_h, b, t0, t1, begin_tile, nblk;  // b: of next_k
    attn_blk k, next_k;
    const attn_blk *blk;
    __device__ __forceinline__ void fetch(uint32_t i)
    {
        const int4 *g = reinterpret_cast<const int4 *>(blk + i);
        int4 *d = reinterpret_cast<int4 *>(&next_k);
        d[0] = g[0];
        d[1] = g[1];
    }
    // s: this CTA's beginning, and the next one's
    __device__ __forceinline__ void begin(const attn_start *s, const attn_blk *list, uint32_t of_block)
    {
        blk = list;
        extra = of_block;
        next_h = s->head;
        b = s->blk;
        begin_tile = s->tile;
        nblk = s->nblk;
        next_k = s->k;
        left = s[1].pos - s->pos;
    }
    __device__ __forceinline__ bool next()
    {
        if (left == 0) return false;
        while (next_k.nt == 0) step();
        k = next_k;
        h = next_h;
        t0 = begin_tile;
        begin_tile = 0;
        if (t0 == 0) left -= extra;
        t1 = (uint32_t)k.nt - t0 < left ? (uint32_t)k.nt : t0 + (uint32_t)left;
        left -= t1 - t0;
        if (left) step();  // a piece that does not end its block is the last
        return true;
    }
    __device__ __forceinline__ void step()
    {
        if (++b == nblk) {
            b = 0;
            ++next_h;
        }
        fetch(b);
    }
    // scratch place of this piece, or -1: the block is all here
    __device__ __forceinline__ int slot() const
    {
        return t0 ? 2 * (int)blockIdx.x : (t1 < (uint32_t)k.nt ? 2 * (int)blockIdx.x + 1 : -1);
    }
};

// ---- many rows --------------------------------------------------------------------------------
// 256 query rows in two tiles of 128 (row r of a tile: token r / G, head r % G of the key head's
// group).  Scores of tile X are in columns X*128 .. of tensor memory; the weights of 64 keys, 16 bits
// wide, take the first half of the same columns and are the left operand of the product with v, which
// adds to columns 256 + X*D ...  While one tile's scores are in the softmax, the tensor cores work
// on the other's, so the softmax has to be as short as a tile's two products (1,024 cycles each way):
// a row belongs to two threads, 64 keys each, which exchange their maxima through shared memory, and
// the product with v begins when half of the weights are there.
// Measured (one GB300, 32/8 heads of 128, causal): 8,192 tokens 366 us, 1,504 TFLOP/s, tensor cores at work
// in 72% of the cycles; about 2,650 cycles for a pair of tiles whose products take 2,048: scores to weights
// 1,250 cycles (exponentials half of them), hand-overs the rest.  Calls of milliseconds meet the power limit.
template <int D, bool E8>
struct rows_cfg {
    static constexpr int kChunks = D / 64;               // 64 elements: a 128-byte row
    static constexpr int kTile = kRowsTile * D * 2;      // bytes of 128 rows
    static constexpr int kStages = (D == 128 ? 5 : 10) - (E8 ? D == 128 ? 1 : 2 : 0);  // of a tile's keys or values
    static constexpr int kCodes = E8 ? (D == 128 ? 2 : 6) : 0;  // tiles as they come, in 8 bits
    static constexpr int kCodeTile = kRowsTile * D;
    // after the tiles: a value per (tile, half, row), pieces, barriers, scales of 16 groups of eight keys, two words
    static constexpr int kCode0 = (2 + kStages) * kTile, kXch = kCode0 + kCodes * kCodeTile;
    static constexpr int kPieces = kXch + 4 * kRowsTile * 4, kBars = kPieces + 2 * 48;
    static constexpr int kScales = kBars + 8 * (26 + 2 * kStages + 2 * kCodes);
    static constexpr int kRefs = kScales + 64 * kCodes;  // of eight tiles, keys and values
    static constexpr int kUp = kRefs + (E8 ? 64 : 0);    // of each query row, the power of two it was multiplied by
    static constexpr int kSmem = kUp + (E8 ? 2 * kRowsTile : 0) + 16;
    static_assert(kSmem <= 227 * 1024, "shared memory of a CTA");
};
// Warps 0-15: softmax (tile, half of the keys, 32 rows); 16: products; 17: copies; 18, 19 make the
// warpgroup whole, whose registers go to the softmax threads: 512 x 104 + 128 x 64 = 640 x 96.
constexpr int kRowsThreads = 640;
// Keys and values in 8 bits: warps 18 to 21 make tiles of halves of them, and zeros of what is behind the sequence; the
// products are of halves whatever the queries' type.  So that these are enough, each tile's largest power of two R
// becomes 2^7 in the tile: the others are exact while they are above 2^-22 R, and off by less than 2^-31 R otherwise.
// The softmax threads multiply scores by R of the keys' tile; values' R is the largest of the piece so far, and as it grows
// the accumulator is scaled.  They hold weights 2^6 times larger, so that those below the row's largest by 2^20 are still
// rounded to 11 bits, and bring each row of bfloat16 queries to 2^14 .. 2^15 by a power of two (k_attn_few8).
// Tiles of bfloat16 would be exact without R, at twice the instructions.  Registers: 512 x 96 + 256 x 48 = 768 x 80, and 20
// to 48 bytes of spill stores.
// Measured (one GB300, 40 suffixes of 1 to 128 tokens over prefixes to 16,384, 32/4 heads of 128): 155 us a call (153 before
// scores beyond kFar were looked after), with two widening warps 170, with tiles of bfloat16 249.  Tensor cores at work in
// 47% of the cycles (16-bit pages: 60%); a copy of the kernel that leaves the widening out takes 18 us less.
constexpr int kRowsWiden = 4;
constexpr float kLift = 6.f;  // of the weights' logarithms
constexpr float kUnlift = 0x1p-6f;
__host__ __device__ constexpr int rows_threads(bool e8) { return e8 ? 768 : kRowsThreads; }

enum { B_QFULL, B_QEMPTY, B_DONE, B_SFULL, B_PREADY = B_SFULL + 2, B_OFULL = B_PREADY + 4, B_OEMPTY = B_OFULL + 2,
       B_PFULL = B_OEMPTY + 2, B_PEMPTY = B_PFULL + 2, B_LREAD = B_PEMPTY + 2, B_QREADY = B_LREAD + 8, B_FULL };

// What the copying warp tells the others of a piece (two of them are kept).
struct rows_piece {
    int row0, ntok, klen, diag;
    int h, t0, n, slot;  // n: key tiles, 0: no more pieces
    int stage, phase;    // of the ring, at its first keys
    int pad[2];
};
static_assert(sizeof(rows_piece) == 48, "shared memory of the pieces");

template <int D, bool BF16, bool E8>
__global__ void __launch_bounds__(rows_threads(E8), 1)
    k_attn_rows(const __grid_constant__ attn_in A, const __grid_constant__ CUtensorMap map_q,
                const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using cfg = rows_cfg<D, E8>;
    static_assert(B_FULL <= 26, "barriers");
    extern __shared__ __align__(1024) unsigned char dyn[];
    volatile rows_piece *piece = reinterpret_cast<volatile rows_piece *>(dyn + cfg::kPieces);
    float(*xch)[kRowsTile] = reinterpret_cast<float(*)[kRowsTile]>(dyn + cfg::kXch);
    uint32_t &tmem_at = *reinterpret_cast<uint32_t *>(dyn + cfg::kSmem - 16);
    int &gave_up = *reinterpret_cast<int *>(dyn + cfg::kSmem - 12);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t sq = cr_smem(dyn), ring = sq + 2 * cfg::kTile;
    const uint32_t bar = sq + cfg::kBars;
    if (sq & 1023u) {  // the swizzled tiles begin at multiples of 1,024 bytes
        cr_wait_previous();  // who waits for this kernel waits for those before it
        if (threadIdx.x == 0) atomicOr(A.status, CR_FLAG_INTERNAL);
        return;
    }
#define BAR(i) (bar + 8u * (uint32_t)(i))
#define FULL(s) BAR(B_FULL + (s))
#define EMPTY(s) BAR(B_FULL + cfg::kStages + (s))
#define CODES(s) BAR(B_FULL + 2 * cfg::kStages + (s))
#define TAKEN(s) BAR(B_FULL + 2 * cfg::kStages + cfg::kCodes + (s))

    if (threadIdx.x == 32) {
        cr_tma_prefetch_map(&map_q);
        cr_tma_prefetch_map(&map_k);
        cr_tma_prefetch_map(&map_v);
    }
    if (threadIdx.x == 0) {
        gave_up = 0;
        cr_bar_init(BAR(B_QFULL), 1);
        cr_bar_init(BAR(B_QEMPTY), 1);
        cr_bar_init(BAR(B_DONE), 1);
        for (int x = 0; x < 2; ++x) {
            cr_bar_init(BAR(B_SFULL + x), 1);
            cr_bar_init(BAR(B_PREADY + 2 * x), 8);
            cr_bar_init(BAR(B_PREADY + 2 * x + 1), 8);
            cr_bar_init(BAR(B_OFULL + x), 1);
            cr_bar_init(BAR(B_OEMPTY + x), 8);
            cr_bar_init(BAR(B_PFULL + x), 1);
            cr_bar_init(BAR(B_PEMPTY + x), E8 ? 17 + kRowsWiden : 17);
        }
        for (int i = 0; i < 8; ++i) cr_bar_init(BAR(B_LREAD + i), 2);
        cr_bar_init(BAR(B_QREADY), 16);
        for (int s = 0; s < cfg::kStages; ++s) {
            cr_bar_init(FULL(s), E8 ? kRowsWiden : 1);
            cr_bar_init(EMPTY(s), 1);
        }
        for (int s = 0; E8 && s < cfg::kCodes; ++s) {
            cr_bar_init(CODES(s), 1 + 16);  // the copies of the tile, and of its 16 scales
            cr_bar_init(TAKEN(s), kRowsWiden);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // query rows that no copy writes (128 is not a multiple of G) are zeros
    if (A.G * A.tq < kRowsTile)
        for (uint32_t i = threadIdx.x; i < 2u * cfg::kTile / 16; i += rows_threads(E8))
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sq + 16 * i), "r"(0));
    cr_fence_async_smem();
    if (warp == 16) cr_tmem_alloc(cr_smem(&tmem_at), 512);
    cr_tc_before();
    __syncthreads();
    cr_tc_after();
    const uint32_t tmem = tmem_at;
    cr_wait_previous();
    if (A.to_pfx) cr_launch_next();  // k_attn_few of the same call gets ready on the SMs that come free

    uint32_t pieces = 0;  // their number so far; they take two places in turn

    if (warp >= 16) {
        if (E8)
            asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        else
            asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    }
    if (warp == 17) {
        // ---- copies ----
        const uint32_t q_bytes = A.G * A.tq * 128 * cfg::kChunks;
        uint32_t stage = 0, phase = 0;
        walk w;
        w.begin(A.start + blockIdx.x, A.blk, A.extra);
        for (;;) {
            const bool more = w.next();
            if (!cr_bar_wait(BAR(B_PEMPTY + (pieces & 1)), ((pieces >> 1) & 1) ^ 1, &gave_up)) goto out;
            if (lane == 0) {
                volatile rows_piece *p = piece + (pieces & 1);
                p->n = more ? (int)(w.t1 - w.t0) : 0;
                if (more) {
                    p->row0 = w.k.row0;
                    p->ntok = w.k.ntok;
                    p->klen = w.k.klen;
                    p->diag = w.k.diag;
                    p->h = (int)w.h;
                    p->t0 = (int)w.t0;
                    p->slot = w.slot();
                    p->stage = (int)stage;
                    p->phase = (int)phase;
                }
                cr_bar_arrive(BAR(B_PFULL + (pieces & 1)));
            }
            __syncwarp();
            if (!more) break;
            if (A.to_pfx && lane == 0) {
                const uint64_t at = (uint64_t)w.k.row0 * A.kv_heads + w.h;
                if (w.t0 == 0) A.first_cta[at] = (int)blockIdx.x;
                if (w.t1 == (uint32_t)w.k.nt) A.last_cta[at] = (int)blockIdx.x;
            }
            const int two = w.k.ntok > (int)A.tq;
            if (!cr_bar_wait(BAR(B_QEMPTY), (pieces & 1) ^ 1, &gave_up)) goto out;
            ++pieces;
            if (lane == 0) cr_bar_expect(BAR(B_QFULL), q_bytes * (1 + two));
            __syncwarp();
            if ((int)lane < cfg::kChunks * (1 + two)) {
                const int x = (int)lane / cfg::kChunks, ch = (int)lane % cfg::kChunks;
                cr_tma_load(sq + x * cfg::kTile + ch * (kRowsTile * 128), &map_q, BAR(B_QFULL), ch * 64, 0, (int)w.h,
                            w.k.row0 + x * (int)A.tq);
            }
            // lane: one box of one column block of a tile
            const uint32_t boxes = kRowsTile >> A.box_log2;
            const uint32_t box = lane & (boxes - 1), ch = lane / boxes;
            const uint32_t at = ch * (kRowsTile * 128) + ((box << A.box_log2) * 128);
            const int32_t *row = A.paged ? A.table + (uint64_t)w.k.kbase * A.max_pages : nullptr;
            if constexpr (E8) {
                // lane: group of eight keys, whose scale it brings; lanes at a box' first group bring the box
                const uint32_t group = lane & 15;
                auto page_of = [&](uint32_t t) {  // n_pages: none
                    const uint32_t at = t * kRowsTile + group * 8;
                    return t < w.t1 && (int)at < w.k.klen ? (uint32_t)row[at >> A.page_log2] : A.n_pages;
                };
                uint32_t next = page_of(w.t0);
                for (uint32_t t = w.t0; t < w.t1; ++t) {
                    const uint32_t key = t * kRowsTile + group * 8, in_page = key & ((1u << A.page_log2) - 1);
                    const uint32_t page = next;
                    next = page_of(t + 1);
                    const bool on = lane < 16 && page < A.n_pages, brings = on && (group * 8 & (A.box_rows - 1)) == 0;
                    const uint32_t bytes = __popc(__ballot_sync(~0u, brings)) * A.box_rows * D;
                    const uint64_t scale = on ? (((uint64_t)page * A.kv_heads + w.h) << A.nb_log2) + (in_page >> A.block_log2) : 0;
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        if (!cr_bar_wait(TAKEN(stage), phase ^ 1, &gave_up)) goto out;
                        if (lane == 0) cr_bar_expect(CODES(stage), bytes);
                        __syncwarp();
                        if (brings)
                            cr_tma_load(sq + cfg::kCode0 + stage * cfg::kCodeTile + group * 8 * D, v ? &map_v : &map_k, CODES(stage), 0,
                                        (int)in_page, (int)w.h, (int)page);
                        if (lane < 16)
                            cr_copy_word(sq + cfg::kScales + stage * 64 + group * 4, (v ? A.v_scale : A.k_scale) + scale, on, CODES(stage));
                        if (++stage == cfg::kCodes) {
                            stage = 0;
                            phase ^= 1;
                        }
                    }
                }
            } else
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                const int key = (int)(t * kRowsTile + (box << A.box_log2));
                // packed keys come as one box; its rows behind the sequence are never used
                const bool on = lane < boxes * cfg::kChunks && (!A.paged || key < w.k.klen);
                int y, pg = 0;
                if (!A.paged) {
                    y = w.k.kbase + key;
                } else {
                    // an ordinary load: k_pages_extend and others of the same chain may still write tables while this
                    // kernel is resident, which only ordinary loads behind the wait above are ordered with
                    if (on) pg = row[(uint32_t)key >> A.page_log2];
                    y = key & ((1 << A.page_log2) - 1);
                }
                const uint32_t bytes = __popc(__ballot_sync(~0u, on)) * A.box_rows * 128;
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    if (!cr_bar_wait(EMPTY(stage), phase ^ 1, &gave_up)) goto out;
                    if (lane == 0) cr_bar_expect(FULL(stage), bytes);
                    __syncwarp();
                    if (on)
                        cr_tma_load(ring + stage * cfg::kTile + at, v ? &map_v : &map_k, FULL(stage), (int)ch * 64, y,
                                    (int)w.h, pg);
                    if (++stage == cfg::kStages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
            }
        }
    } else if (warp == 16) {
        // ---- products ----
        const uint32_t me = cr_elect();
        const uint32_t id_s = cr_idesc(BF16 && !E8, 128, 128, false), id_o = cr_idesc(BF16 && !E8, 128, D, true);
        uint32_t stage = 0, phase = 0, pphase[2] = {0, 0}, ophase[2] = {0, 0};
        auto scores = [&](int x, uint32_t st) {
            const uint32_t a = sq + x * cfg::kTile, b = ring + st * cfg::kTile;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const uint32_t off = (i / 4) * (kRowsTile * 128) + (i % 4) * 32;
                cr_mma_ss(tmem + x * 128, cr_sdesc(a + off, 16, 1024), cr_sdesc(b + off, 16, 1024), id_s, i > 0, me);
            }
        };
        // 16 keys a step: of each thread's 64 keys the first half (part 0), then the second
        auto values = [&](int x, uint32_t st, int part, bool first) {
            const uint32_t b = ring + st * cfg::kTile;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = (e >> 1) * 4 + part * 2 + (e & 1);
                cr_mma_ts(tmem + 256 + x * D, tmem + x * 128 + (e >> 1) * 64 + (part * 2 + (e & 1)) * 8,
                          cr_sdesc(b + i * 2048, kRowsTile * 128, 1024), id_o, !(first && part == 0 && e == 0), me);
            }
        };
        auto forward = [&]() {
            if (++stage == cfg::kStages) {
                stage = 0;
                phase ^= 1;
            }
        };
        // weights x values of a tile, then the next scores
        auto turn = [&](int x, uint32_t vs, bool first, bool more) {
            if (first) {
                if (!cr_bar_wait(BAR(B_OEMPTY + x), ophase[x] ^ 1, &gave_up)) return false;
                ophase[x] ^= 1;
            }
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                if (!cr_bar_wait(BAR(B_PREADY + 2 * x + part), pphase[x], &gave_up)) return false;
                cr_tc_after();
                values(x, vs, part, first);
            }
            pphase[x] ^= 1;
            if (more) {
                scores(x, stage);
                cr_tc_commit(BAR(B_SFULL + x), me);
            } else {
                cr_tc_commit(BAR(B_OFULL + x), me);
            }
            return true;
        };
        for (;; ++pieces) {
            if (!cr_bar_wait(BAR(B_PFULL + (pieces & 1)), (pieces >> 1) & 1, &gave_up)) goto out;
            const volatile rows_piece *p = piece + (pieces & 1);
            const uint32_t n = __shfl_sync(~0u, p->n, 0);
            const bool two = __shfl_sync(~0u, p->ntok, 0) > (int)A.tq;
            if (lane == 0) cr_bar_arrive(BAR(B_PEMPTY + (pieces & 1)));
            if (n == 0) break;
            if (!cr_bar_wait(BAR(E8 && BF16 ? B_QREADY : B_QFULL), pieces & 1, &gave_up)) goto out;
            if (!cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
            cr_tc_after();
            scores(0, stage);
            cr_tc_commit(BAR(B_SFULL), me);
            if (two) {
                scores(1, stage);
                cr_tc_commit(BAR(B_SFULL + 1), me);
            }
            cr_tc_commit(EMPTY(stage), me);
            if (n == 1) cr_tc_commit(BAR(B_QEMPTY), me);
            forward();
            for (uint32_t j = 0; j < n; ++j) {
                const bool more = j + 1 < n;
                const uint32_t vs = stage;
                if (!cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
                forward();
                if (more && !cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
                if (!turn(0, vs, j == 0, more)) goto out;
                if (two && !turn(1, vs, j == 0, more)) goto out;
                cr_tc_commit(EMPTY(vs), me);
                if (more) {
                    cr_tc_commit(EMPTY(stage), me);
                    forward();
                }
                if (j + 2 == n) cr_tc_commit(BAR(B_QEMPTY), me);
            }
        }
        cr_tc_commit(BAR(B_DONE), me);  // the shared memory is in use until the last product has ended
        cr_bar_wait(BAR(B_DONE), 0, &gave_up);
    } else if (E8 && warp >= 18 && warp < 18 + kRowsWiden) {
        // ---- tiles of halves: a lane widens rows of its own ----
        uint32_t stage = 0, phase = 0, code = 0, cphase = 0, tile = 0;
        for (;; ++pieces) {
            if (!cr_bar_wait(BAR(B_PFULL + (pieces & 1)), (pieces >> 1) & 1, &gave_up)) goto out;
            const volatile rows_piece *p = piece + (pieces & 1);
            const int n = p->n;
            int left = p->klen - p->t0 * kRowsTile;  // keys from the tile's first on
            __syncwarp();
            if (lane == 0) cr_bar_arrive(BAR(B_PEMPTY + (pieces & 1)));
            if (n == 0) break;
            float top = 0.f;  // values' largest power so far
            for (int j = 0; j < 2 * n; ++j) {
                if (!cr_bar_wait(CODES(code), cphase, &gave_up)) goto out;
                const uint32_t sc = sq + cfg::kScales + code * 64;
                uint32_t r;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(sc + (lane & 15) * 4));
                float ref = __uint_as_float(__reduce_max_sync(~0u, r));
                if (j & 1) ref = top = fmaxf(top, ref);
                if (ref == 0.f) ref = 1.f;  // no keys
                const float per = 128.f / ref;
                const bool whole = left >= kRowsTile && __all_sync(~0u, r != 0);  // a scale of 0: no page
                if (!cr_bar_wait(EMPTY(stage), phase ^ 1, &gave_up)) goto out;
                if (warp == 18 && lane == 0)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(sq + cfg::kRefs + (j & 1) * 32 + (tile & 7) * 4), "f"(ref * 0x1p-7f)
                                 : "memory");
                const uint32_t row = (warp - 18) * 32 + lane;
                float scale;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(scale) : "r"(sc + (row >> 3) * 4));
                const __half2 f = __float2half2_rn(scale * per);
                const uint32_t src = sq + cfg::kCode0 + code * cfg::kCodeTile + row * D, turn = D == 128 ? row & 7 : (row >> 1) & 3;
                const uint32_t dst = ring + stage * cfg::kTile + row * 128;
                const bool none = !whole && ((int)row >= left || scale == 0.f);
#pragma unroll
                for (uint32_t c0 = 0; c0 < D / 16; c0 += 4) {
                    uint32_t q[4][4];
#pragma unroll
                    for (uint32_t c = 0; c < 4; ++c)
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(q[c][0]), "=r"(q[c][1]), "=r"(q[c][2]), "=r"(q[c][3])
                                     : "r"(src + (((c0 + c) ^ turn) << 4)));
                    if (none) {
#pragma unroll
                        for (uint32_t c = 0; c < 4; ++c) q[c][0] = q[c][1] = q[c][2] = q[c][3] = 0;
                    }
#pragma unroll
                    for (uint32_t c = 0; c < 4; ++c) {
                        uint32_t o[8];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            cr_e4m3_halves(q[c][e], o[2 * e], o[2 * e + 1]);
#pragma unroll
                            for (int h = 2 * e; h < 2 * e + 2; ++h) {
                                const __half2 y = __hmul2(*reinterpret_cast<const __half2 *>(&o[h]), f);
                                o[h] = *reinterpret_cast<const uint32_t *>(&y);
                            }
                        }
                        const uint32_t to = dst + (c0 >> 2) * (kRowsTile * 128), u = c * 2;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((u ^ (row & 7)) << 4)), "r"(o[0]),
                                     "r"(o[1]), "r"(o[2]), "r"(o[3])
                                     : "memory");
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((u + 1) ^ (row & 7)) << 4)), "r"(o[4]),
                                     "r"(o[5]), "r"(o[6]), "r"(o[7])
                                     : "memory");
                    }
                }
                cr_fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    cr_bar_arrive(FULL(stage));
                    cr_bar_arrive(TAKEN(code));
                }
                if (++stage == cfg::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
                if (++code == cfg::kCodes) {
                    code = 0;
                    cphase ^= 1;
                }
                if (j & 1) {
                    left -= kRowsTile;
                    ++tile;
                }
            }
        }
    } else if (warp < 16) {
        // ---- softmax: two threads a row ----
        if (E8)
            asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
        else
            asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int x = (int)(warp >> 3), half = (int)(warp >> 2) & 1;
        const uint32_t row = (warp & 3) * 32 + lane;
        // this warp's lanes of tensor memory, its scores (and weights), its columns of the accumulator
        const uint32_t ts = tmem + ((warp & 3) << 21) + x * 128 + half * 64;
        const uint32_t to = tmem + ((warp & 3) << 21) + 256 + x * D + half * (D / 2);
        const uint32_t pair = 1 + x * 4 + (warp & 3);  // barrier of the two warps that share rows
        // 8 bits: sums are scaled by powers of two as they come, that of A.c among them, which leaves less than 2
        const float c = E8 ? A.c_rest : A.c, c_far = E8 ? 1.f : A.c_pow;
        const int tok = x * (int)A.tq + (int)(row / A.G), hd = row < A.G * A.tq ? (int)(row % A.G) : -1;
        uint32_t sphase = 0;
        // The other half's value of this row.  The next value is written only after the other warp has read this
        // one: the next scores come after both warps' weights, and a piece's sums have B_LREAD before and after them.
        // Between two meetings there is always a wait with a limit, where a warp may leave (then it releases its
        // partner once).
        auto meet = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory"); };
        auto exchange = [&](float v) {
            xch[x * 2 + half][row] = v;
            meet();
            return xch[x * 2 + (half ^ 1)][row];
        };
        // 8 bits: a piece's bfloat16 queries as halves, each row brought to 2^14 .. 2^15; two lanes a row, and the two
        // warps that share 32 rows half of them each.  Done as soon as the piece before has no more weights to make, so
        // that its result is written while the products go on (after that result: 0.5 us a piece more).
        float next_c = A.c_pow;
        uint32_t tile = 0;  // 8 bits: key tiles so far
        auto halve = [&](uint32_t i) {
            if (!cr_bar_wait(BAR(B_PFULL + (i & 1)), (i >> 1) & 1, &gave_up)) return false;
            const volatile rows_piece *p = piece + (i & 1);
            if (p->n == 0) return true;
            if (!cr_bar_wait(BAR(B_QFULL), i & 1, &gave_up)) return false;  // also who has no rows: no phase is left out
            if (x == 0 || p->ntok > (int)A.tq) {
                constexpr int kC = D / 16;  // chunks of eight elements
                const uint32_t r = (warp & 3) * 32 + half * 16 + (lane & 15), h = lane >> 4, turn = r & (D == 128 ? 7 : 3);
                const uint32_t at = sq + x * cfg::kTile + r * 128 + (D == 128 ? h * (kRowsTile * 128) : ((h * 4) ^ (r & 4)) * 16);
                uint32_t q[kC][4], most = 0;
#pragma unroll
                for (uint32_t k = 0; k < kC; ++k) {
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(q[k][0]), "=r"(q[k][1]), "=r"(q[k][2]), "=r"(q[k][3])
                                 : "r"(at + ((k ^ turn) << 4)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = max(most, max(q[k][e] << 16 & 0x7fffffffu, q[k][e] & 0x7fff0000u));
                }
                most = max(most, __shfl_xor_sync(~0u, most, 16));
                const int up = max(-113, min(113, 14 + 127 - (int)(most >> 23)));
                const float f = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
                for (uint32_t k = 0; k < kC; ++k) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        q[k][e] = cr_pack16<false>(__uint_as_float(q[k][e] << 16) * f, __uint_as_float(q[k][e] & 0xffff0000u) * f);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + ((k ^ turn) << 4)), "r"(q[k][0]), "r"(q[k][1]),
                                 "r"(q[k][2]), "r"(q[k][3])
                                 : "memory");
                }
                const uint32_t ups = sq + cfg::kUp + x * kRowsTile;
                if (h == 0) asm volatile("st.shared.b8 [%0], %1;" ::"r"(ups + r), "r"(up) : "memory");
                cr_fence_async_smem();
                meet();
                int mine;
                asm volatile("ld.shared.s8 %0, [%1];" : "=r"(mine) : "r"(ups + row) : "memory");
                next_c = A.c_pow * __uint_as_float((uint32_t)(127 - mine) << 23);
            }
            __syncwarp();
            if (lane == 0) cr_bar_arrive(BAR(B_QREADY));
            return true;
        };
        if (E8 && BF16 && !halve(0)) goto left;
        for (uint32_t ophase = 0;; ++pieces) {
            if (!cr_bar_wait(BAR(B_PFULL + (pieces & 1)), (pieces >> 1) & 1, &gave_up)) goto left;
            const volatile rows_piece *p = piece + (pieces & 1);
            const int n = p->n;
            if (n == 0) break;
            if (x == 1 && p->ntok <= (int)A.tq) {
                __syncwarp();
                if (lane == 0) cr_bar_arrive(BAR(B_PEMPTY + (pieces & 1)));
                tile += (uint32_t)n;
                if (E8 && BF16 && !halve(pieces + 1)) goto left;
                continue;
            }
            const float cq = next_c;
            float unit = 0.f;  // of the accumulator
            // keys that this row sees, from the first tile's on; the tile with the sequence's end
            int seen = p->klen - p->t0 * kRowsTile - half * 64;
            const int tail = !E8 && x == 0 && half < cfg::kChunks ? (p->klen >> 7) - p->t0 : -1;
            if (A.causal) seen = min(seen, p->diag - p->t0 * kRowsTile - half * 64 + tok + 1);
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < n; ++j, seen -= kRowsTile) {
                if (!cr_bar_wait(BAR(B_SFULL + x), sphase, &gave_up)) goto left;
                sphase ^= 1;
                cr_tc_after();
                uint32_t s[64];
                cr_tmem_ld(ts, s);
                cr_tmem_ld(ts + 32, s + 32);
                cr_tmem_ld_wait();
                if (__any_sync(~0u, seen < 64)) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) s[i] = i < seen ? s[i] : 0xff800000u;
                }
                float mx[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mx[i] = __uint_as_float(s[i]);
#pragma unroll
                    for (int e = 4; e < 60; e += 8)
                        mx[i] = cr_max3(mx[i], __uint_as_float(s[e + i]), __uint_as_float(s[e + 4 + i]));
                    mx[i] = fmaxf(mx[i], __uint_as_float(s[60 + i]));
                }
                float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                float ct = 1.f, now = 0.f;
                if (E8) {
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ct) : "r"(sq + cfg::kRefs + (tile & 7) * 4));
                    // above 0, as what it multiplies may be masked, minus infinity; sums are below 2^40, so that scores which
                    // this enlarges are still below 2^-86
                    ct = fmaxf(ct * cq, 0x1p-126f);
                }
                top = fmaxf(top, exchange(top));
                if (E8) top *= ct;
                // The maximum may lag by 2^8: weights stay below 2^8, sums below 2^31, and the
                // accumulator is scaled a few times per row instead of at every tile.
                const bool grow = j == 0 || !(E8 ? (top - m) * c < 8.f || top == m : (top - m) * c <= 8.f || top == m);
                if (__any_sync(~0u, grow)) {
                    const float m_new = fmaxf(m, top);
                    if (j > 0) {
                        const float f = m_new == m ? 1.f : cr_exp2((m - m_new) * c);
                        l *= f;
#pragma unroll 1
                        for (int i = 0; i < D / 2; i += 16) {
                            uint32_t o[16];
                            cr_tmem_ld16(to + i, o);
                            cr_tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            cr_tmem_st16(to + i, o);
                        }
                        cr_tmem_st_wait();
                    }
                    m = m_new;
                }
                // keys behind the sequence's end have weight zero, but what stands there may be
                // no number: their rows of v become zeros
                if (j == tail) {
                    const uint32_t at = (uint32_t)p->stage + 2 * j + 1;
                    const uint32_t st = at % cfg::kStages, ph = (uint32_t)p->phase ^ ((at / cfg::kStages) & 1);
                    if (!cr_bar_wait(FULL(st), ph, &gave_up)) goto left;
                    if ((int)row >= (p->klen & (kRowsTile - 1))) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(
                                             ring + st * cfg::kTile + half * (kRowsTile * 128) + row * 128 + i * 16),
                                         "r"(0)
                                         : "memory");
                    }
                    cr_fence_async_smem();
                }
                const float by = fabsf(m) > (E8 ? kFar : A.far) ? c_far : c;
                const unsigned long long c2 = E8 ? cr_pair(ct * by, ct * by) : cr_pair(by, by);
                constexpr float lift = E8 ? kLift : 0.f;
                const float off = m == -INFINITY ? lift : E8 ? fmaf(-m, by, lift) : -m * by;
                if (E8) {
                    const uint32_t at = 2 * tile + 1;  // the values' R
                    if (!cr_bar_wait(FULL(at % cfg::kStages), (at / cfg::kStages) & 1, &gave_up)) goto left;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(now) : "r"(sq + cfg::kRefs + 32 + (tile & 7) * 4));
                    ++tile;
                }
                const unsigned long long off2 = cr_pair(off, off);
                unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int i = part * 32 + 2 * e;
                        float a, b;
                        cr_unpair(cr_fma2(cr_pair(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2, off2), a, b);
                        a = cr_exp2(a);
                        b = cr_exp2(b);
                        sum[e & 1] = cr_add2(sum[e & 1], cr_pair(a, b));
                        w[e] = cr_pack16<BF16 && !E8>(a, b);
                    }
                    cr_tmem_st16(ts + part * 16, w);
                    if (E8 && part == 0) {
                        if (now != unit && j > 0) {
                            const float f = unit / now;
#pragma unroll 1
                            for (int i = 0; i < D / 2; i += 16) {
                                uint32_t o[16];
                                cr_tmem_ld16(to + i, o);
                                cr_tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                cr_tmem_st16(to + i, o);
                            }
                        }
                        unit = now;
                    }
                    cr_tmem_st_wait();
                    cr_tc_before();
                    __syncwarp();
                    if (lane == 0) cr_bar_arrive(BAR(B_PREADY + 2 * x + part));
                }
                float s0, s1;
                cr_unpair(cr_add2(sum[0], sum[1]), s0, s1);
                l += s0 + s1;
            }
            // ---- the piece's result ----
            // While the last product is under way: the sums meet where the maxima did, once both warps have read those,
            // and whatever else the result needs (0.5 to 1.5% of a call against doing it after that product).
            __syncwarp();
            if (lane == 0) cr_bar_arrive(BAR(B_LREAD + pair - 1));
            if (!cr_bar_wait(BAR(B_LREAD + pair - 1), 0, &gave_up)) goto left;
            const float l2 = exchange(l);
            __syncwarp();
            if (lane == 0) cr_bar_arrive(BAR(B_LREAD + pair - 1));
            l = half ? l2 + l : l + l2;
            if (E8 && BF16 && !halve(pieces + 1)) goto left;
            const bool valid = hd >= 0 && tok < p->ntok;
            const int slot = p->slot;
            const int head = p->h * (int)A.G + hd;
            const uint64_t tk = (uint64_t)(p->row0 + tok);
            const float inv = l == 0.f ? 0.f : E8 ? unit / l : 1.f / l;
            if (!cr_bar_wait(BAR(B_OFULL + x), ophase, &gave_up)) goto left;
            ophase ^= 1;
            cr_tc_after();
            if (slot >= 0) {
                constexpr int RP = 2 * kRowsTile;  // rows of a piece
                const uint32_t r = x * kRowsTile + row;
                float4 *dst = reinterpret_cast<float4 *>(A.part) + ((uint64_t)slot * (D / 4) + half * (D / 8)) * RP + r;
#pragma unroll 1
                for (int i = 0; i < D / 2; i += 16) {
                    uint32_t o[16];
                    cr_tmem_ld16(to + i, o);
                    cr_tmem_ld_wait();
                    if (E8) {  // sums of weights as they are: values near the type's largest leave no room for more
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * (unit * kUnlift));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        dst[(i / 4 + e) * RP] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]),
                                                            __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                }
                if (half == 0)
                    reinterpret_cast<float2 *>(A.part_ml)[(uint64_t)slot * RP + r] =
                        make_float2(m == -INFINITY ? m : E8 ? fmaf(m, c, -kLift) + kLift : m * c, E8 ? l * kUnlift : l);
            } else {
                if (!A.to_pfx && A.o_wide && A.head_dim == D) {
                    // Lanes of a group of C hold C chunks of 32 bytes of a row each; the chunks change places, so that a
                    // store of the group writes C chunks of a row side by side: 32 rows at once would be 32 lines
                    // (twelve prompts of up to 4,096 tokens: 244 us with a row per lane, 237 so).
                    constexpr int C = D / 32;
                    uint32_t v[8 * C];
#pragma unroll
                    for (int q = 0; q < C; ++q) {
                        uint32_t o[16];
                        cr_tmem_ld16(to + 16 * q, o);
                        cr_tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            v[8 * q + e] = l == 0.f ? 0u
                                                    : cr_pack16<BF16>(__uint_as_float(o[2 * e]) * inv,
                                                                      __uint_as_float(o[2 * e + 1]) * inv);
                    }
#pragma unroll
                    for (int b = 1; b < C; b *= 2)
#pragma unroll
                        for (int q = 0; q < C; ++q) {
                            if (q & b) continue;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                uint32_t &lo = v[8 * q + e], &hi = v[8 * (q + b) + e];
                                const uint32_t got = __shfl_xor_sync(~0u, lane & b ? lo : hi, b);
                                if (lane & b)
                                    lo = got;
                                else
                                    hi = got;
                            }
                        }
                    uint16_t *dst = static_cast<uint16_t *>(A.o) + half * (D / 2) + (lane & (C - 1)) * 16;
                    const uint64_t at = valid ? tk * A.o_token + head * A.o_head : ~0ull;
#pragma unroll
                    for (int q = 0; q < C; ++q) {
                        const uint64_t its = __shfl_sync(~0u, at, (int)((lane & ~(C - 1)) | q));
                        if (its != ~0ull) cr_store32(dst + its, v + 8 * q);
                    }
                } else {
#pragma unroll 1
                    for (int i = 0; i < D / 2; i += 16) {
                        uint32_t o[16];
                        cr_tmem_ld16(to + i, o);
                        cr_tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv);
                        const int d0 = half * (D / 2) + i;
                        if (!valid) continue;
                        if (A.to_pfx) {
                            float *dst = A.pfx + (tk * A.q_heads + head) * D + d0;
                            cr_store32(dst, o);
                            cr_store32(dst + 8, o + 8);
                        } else {
                            uint16_t *dst = static_cast<uint16_t *>(A.o) + tk * A.o_token + head * A.o_head + d0;
                            uint32_t v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                v[e] = cr_pack16<BF16>(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
                            if (A.o_wide && d0 + 16 <= (int)A.head_dim) {
                                cr_store32(dst, v);
                            } else {
                                if (d0 < (int)A.head_dim) *reinterpret_cast<uint4 *>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
                                if (d0 + 8 < (int)A.head_dim)
                                    *reinterpret_cast<uint4 *>(dst + 8) = make_uint4(v[4], v[5], v[6], v[7]);
                            }
                        }
                    }
                }
                if (valid && half == 0) {
                    const float lse2 = l == 0.f ? -INFINITY : (E8 ? fmaf(m, c, -kLift) : m * c) + log2f(l);
                    if (A.to_pfx)
                        A.pfx_lse[tk * A.q_heads + head] = lse2;
                    else if (A.lse)
                        A.lse[tk * A.q_heads + head] = lse2 * 0.693147180559945309f;
                }
            }
            if (!cr_bar_wait(BAR(B_LREAD + pair - 1), 1, &gave_up)) goto left;
            cr_tc_before();
            __syncwarp();
            if (lane == 0) {
                cr_bar_arrive(BAR(B_OEMPTY + x));
                cr_bar_arrive(BAR(B_PEMPTY + (pieces & 1)));
            }
        }
    left:
        // a wait that has given up: the other warp of the pair must not wait for this one
        if (gave_up) asm volatile("bar.arrive %0, 64;" ::"r"(pair) : "memory");
    }
out:
    __syncwarp();
    if (gave_up) {  // let the copies and products that are under way end
        if (threadIdx.x == 0) atomicOr(A.status, CR_FLAG_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    cr_tc_before();
    __syncthreads();
    cr_launch_next();
    if (warp == 16) {
        cr_tc_after();
        cr_tmem_free(tmem, 512);
    }
#undef FULL
#undef EMPTY
#undef CODES
#undef TAKEN
#undef BAR
}

// ---- joining pieces ---------------------------------------------------------------------------
// Bound by the latency of its dependent reads: about 3 us for two to eight pieces a block.
// 256 threads join 16 rows by D columns: thread (row threadIdx % 16, columns 4 (threadIdx / 16 + 16 x) ..) adds up n
// pieces of its row, ml(i) the maximum and sum of piece i, data(i, column / 4) four columns of it.  The first pieces'
// columns are on their way while the weights are made.
struct join_shared {
    float wgt[32][16], red[16][16];
};
template <int kPer, typename ML, typename DATA>
__device__ __forceinline__ void join_pieces(uint32_t n, ML ml, DATA data, join_shared &S, float &m, float &l, float4 *o)
{
    const uint32_t col = threadIdx.x & 15, grp = threadIdx.x >> 4;
    float4 v[4][kPer];
    auto load = [&](uint32_t i0) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < kPer; ++x)
                v[i][x] = i0 + i < n ? data(i0 + i, grp + 16 * x) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    load(0);
    float2 mine = make_float2(-INFINITY, 0.f);
    if (grp < n) mine = ml(grp);
    m = mine.x;
    for (uint32_t i = grp + 16; i < n; i += 16) m = fmaxf(m, ml(i).x);
    S.red[grp][col] = m;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, S.red[e][col]);
    l = 0.f;
#pragma unroll
    for (int x = 0; x < kPer; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t i0 = 0; i0 < n; i0 += 32) {
        if (i0) __syncthreads();
        for (uint32_t i = grp; i < 32; i += 16) {
            const float2 q = i0 + i == grp ? mine : (i0 + i < n ? ml(i0 + i) : make_float2(-INFINITY, 0.f));
            const float f = q.x == -INFINITY ? 0.f : cr_exp2(q.x - m);
            S.wgt[i][col] = f;
            l += q.y * f;
        }
        __syncthreads();
        const uint32_t ni = min(32u, n - i0);
        for (uint32_t j = 0; j < ni; j += 4) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const float f = S.wgt[j + i][col];
                if (f == 0.f) continue;  // sees none of these keys
#pragma unroll
                for (int x = 0; x < kPer; ++x) {
                    o[x].x += v[i][x].x * f;
                    o[x].y += v[i][x].y * f;
                    o[x].z += v[i][x].z * f;
                    o[x].w += v[i][x].w * f;
                }
            }
            load(i0 + j + 4);
        }
    }
    __syncthreads();  // red may still be read
    S.red[grp][col] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) l += S.red[e][col];
    __syncthreads();
}

// Where the i-th piece of a block lies that CTA `first` began.
__device__ __forceinline__ uint64_t piece_slot(uint32_t first, uint32_t i) { return i == 0 ? 2ull * first + 1 : 2ull * (first + i); }

// A row's result.
template <int kPer, bool BF16>
__device__ __forceinline__ void join_write(const attn_in &A, uint64_t token, uint32_t head, float m, float l, const float4 *o)
{
    const uint32_t grp = threadIdx.x >> 4;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
        const uint32_t d = 4 * (grp + 16 * x);
        if (d < A.head_dim)
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.o) + token * A.o_token + head * A.o_head + d) =
                make_uint2(cr_pack16<BF16>(o[x].x * inv, o[x].y * inv), cr_pack16<BF16>(o[x].z * inv, o[x].w * inv));
    }
    if (grp == 0 && A.lse)
        A.lse[token * A.q_heads + head] = (l == 0.f ? -INFINITY : m + log2f(l)) * 0.693147180559945309f;
}

// Joins the blocks that several CTAs worked on, 16 rows of one at a time.  Pieces lie in scratch as [D / 4][RP rows][4].
template <int D, bool BF16, int RP>
__global__ void __launch_bounds__(256) k_attn_join(const __grid_constant__ attn_in A)
{
    __shared__ join_shared S;
    cr_launch_next();
    cr_wait_previous();
    const bool own = RP == 16 && A.own_list;  // no list: every stretch but the first may join pieces
    const uint32_t items = (own ? A.ncta - 1 : A.joins[0]) * (RP / 16);
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t c = own ? 1 + item : A.joins[1 + item / (RP / 16)], r = item % (RP / 16) * 16 + (threadIdx.x & 15);
        const attn_start s = A.start[c];
        if (own && s.pieces == 0) continue;
        bool valid;
        uint32_t head;
        uint64_t tk = (uint64_t)s.k.row0;
        if (RP == 16) {
            head = s.head / A.nsub * A.G + s.head % A.nsub * 16 + r;
            valid = s.head % A.nsub * 16 + r < A.G;
        } else {
            const uint32_t x = r / kRowsTile, rr = r % kRowsTile, tok = x * A.tq + rr / A.G;
            valid = rr < A.G * A.tq && (int)tok < s.k.ntok;
            head = s.head * A.G + rr % A.G;
            tk += tok;
        }
        if (!__syncthreads_or(valid)) continue;  // the second tile is not in use
        float m, l;
        float4 o[D / 64];
        join_pieces<D / 64>(
            s.pieces,
            [&](uint32_t i) { return reinterpret_cast<const float2 *>(A.part_ml)[piece_slot(c - 1, i) * RP + r]; },
            [&](uint32_t i, uint32_t d4) {
                return reinterpret_cast<const float4 *>(A.part)[(piece_slot(c - 1, i) * (D / 4) + d4) * RP + r];
            },
            S, m, l, o);
        if (valid) join_write<D / 64, BF16>(A, tk, head, m, l, o);
    }
}

// Joins everything that a single token's heads have: the pieces of its own keys (or its place, where one CTA had them
// all) and those of its group's shared prefix.  blockIdx: (entry, 16 rows of a key head).
template <int D, bool BF16>
__global__ void __launch_bounds__(256)
    k_attn_decode_join(const __grid_constant__ attn_in F, const __grid_constant__ attn_in R)
{
    __shared__ join_shared S;
    cr_launch_next();
    cr_wait_previous();
    const uint32_t e = blockIdx.x, h = blockIdx.y, kv = h / F.nsub, sub = h % F.nsub;
    const uint64_t own = (uint64_t)e * F.few_heads + h;
    // groups that are not ascending, and waits that have given up, leave some of these unset: no index passes its array
    // all the same
    const int row0 = clampi(R.of_token[e], 0, (int)e);
    const cr_cta_span of_own = cr_marked_ctas(F.first_cta[own], F.last_cta[own], (int)F.ncta);
    const bool shared = F.blk[e].lo > 0;   // else row0 means nothing
    if (of_own.n == 1 && !shared) return;  // written already
    const uint32_t r = threadIdx.x & 15;
    const bool valid = sub * 16 + r < F.G;
    const uint32_t head = kv * F.G + sub * 16 + r;
    const uint64_t oh = (uint64_t)e * F.q_heads + head;
    const uint32_t f0 = (uint32_t)of_own.first, nf = of_own.n;
    uint32_t r0 = 0, nr = 0, rr = 0;
    if (shared) {
        const uint64_t at = (uint64_t)row0 * R.kv_heads + kv;
        const cr_cta_span of_prefix = cr_marked_ctas(R.first_cta[at], R.last_cta[at], (int)R.ncta);
        r0 = (uint32_t)of_prefix.first;
        nr = of_prefix.n;
        const uint32_t t = min(e - (uint32_t)row0, 2 * R.tq - 1);  // token of the prefix' block
        rr = t / R.tq * kRowsTile + t % R.tq * R.G + sub * 16 + r;
    }
    float m, l;
    float4 o[D / 64];
    join_pieces<D / 64>(
        nf + nr,
        [&](uint32_t i) {
            if (!valid) return make_float2(-INFINITY, 0.f);
            if (i < nf)
                return nf == 1 ? reinterpret_cast<const float2 *>(F.own_ml)[own * 16 + r]
                               : reinterpret_cast<const float2 *>(F.part_ml)[piece_slot(f0, i) * 16 + r];
            return nr == 1 ? make_float2(F.pfx_lse[oh], 1.f)
                           : reinterpret_cast<const float2 *>(R.part_ml)[piece_slot(r0, i - nf) * (2 * kRowsTile) + rr];
        },
        [&](uint32_t i, uint32_t d4) {
            if (!valid) return make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < nf)
                return nf == 1 ? reinterpret_cast<const float4 *>(F.own)[(own * (D / 4) + d4) * 16 + r]
                               : reinterpret_cast<const float4 *>(F.part)[(piece_slot(f0, i) * (D / 4) + d4) * 16 + r];
            return nr == 1 ? *reinterpret_cast<const float4 *>(F.pfx + oh * D + 4 * d4)
                           : reinterpret_cast<const float4 *>(
                                 R.part)[(piece_slot(r0, i - nf) * (D / 4) + d4) * (2 * kRowsTile) + rr];
        },
        S, m, l, o);
    if (valid) join_write<D / 64, BF16>(F, e, head, m, l, o);
}

// ---- few rows ---------------------------------------------------------------------------------
// One token's query heads of a key head, 16 at most.  Here the bytes of k and v are the bound
// (each is used for a few rows only), so the small register-operand products do: four warps take
// 16 keys each of a tile of 64 that a fifth warp's copies bring, with the softmax state of the
// rows in every warp, joined at the piece's end.  The next piece's queries are copied meanwhile.
// Two CTAs an SM with 96 KB of copies in flight each; measured: 128 contexts of 4,160 tokens, 64/8 heads of
// 128, pages of 16 tokens: 357 us a call, 6.1 TB/s (a copy runs at 6.8); pages of 64 tokens 2% less.
template <int D>
struct few_cfg {
    static constexpr int kChunks = D / 64;
    static constexpr int kTile = kFewTile * D * 2;       // bytes of 64 keys
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kQ = 16 * D * 2;                // bytes of 16 query rows
    static constexpr int kJoin = kFewWarps * 8 * 64 * 4; // eight rows, 64 columns of every warp
    static constexpr int kSmem = kStages * 2 * kTile + kQ + kJoin + 1024;
};
constexpr int kFewThreads = 32 * (kFewWarps + 1);

template <bool BF16>
__device__ __forceinline__ void mma16816(float *d, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    if (BF16)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void ldsm4(uint32_t *r, uint32_t addr)
{
    if (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
}

template <int D, bool BF16, bool WIDE>
__global__ void __launch_bounds__(kFewThreads, 2)
    k_attn_few(const __grid_constant__ attn_in A, const __grid_constant__ CUtensorMap map_q,
               const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using cfg = few_cfg<D>;
    extern __shared__ unsigned char dyn[];
    __shared__ __align__(8) unsigned long long bars[2 * cfg::kStages + 3];
    __shared__ float2 join_ml[kFewWarps][16];
    __shared__ int gave_up;
    __shared__ own_list list;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = cr_smem(dyn), ring = (base + 1023u) & ~1023u, sq = ring + cfg::kStages * 2 * cfg::kTile;
    float *join = reinterpret_cast<float *>(dyn + (sq - base) + cfg::kQ);
    const uint32_t bar = cr_smem(bars);
#define FULL(s) (bar + 8u * (s))
#define EMPTY(s) (bar + 8u * (cfg::kStages + (s)))
#define QFULL (bar + 8u * (2 * cfg::kStages))
#define QEMPTY (bar + 8u * (2 * cfg::kStages + 1))
#define JOIN (bar + 8u * (2 * cfg::kStages + 2))

    if (threadIdx.x == 32) {
        cr_tma_prefetch_map(&map_q);
        cr_tma_prefetch_map(&map_k);
        cr_tma_prefetch_map(&map_v);
    }
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int s = 0; s < cfg::kStages; ++s) {
            cr_bar_init(FULL(s), 1);
            cr_bar_init(EMPTY(s), kFewWarps);
        }
        cr_bar_init(QFULL, 1);
        cr_bar_init(QEMPTY, kFewWarps);
        cr_bar_init(JOIN, kFewWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (uint32_t i = threadIdx.x; i < cfg::kQ / 16; i += kFewThreads)  // rows that no copy writes
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sq + 16 * i), "r"(0));
    cr_fence_async_smem();
    __syncthreads();
    // After k_attn_rows of the same call this one needs nothing of it, but it does read what was written before that
    // began (the list of work, tables, pages), and only the wait makes any of it visible here.
    cr_wait_previous();
    cr_launch_next();

    walk w;
    plan_cut cut;
    if (A.own_list) {
        if (warp == kFewWarps) cut = make_list(A.plan, &list, A.status);
        __syncthreads();
        w.begin(list.start, list.blk, A.extra);
    } else {
        w.begin(A.start + blockIdx.x, A.blk, A.extra);
    }
    uint32_t stage = 0, phase = 0, qphase = 0;
    if (warp == kFewWarps) {
        // ---- copies: a lane brings one box of one column block, keys and values ----
        const uint32_t boxes = kFewTile >> A.box_log2;
        const uint32_t box = lane & (boxes - 1), ch = lane / boxes;
        while (w.next()) {
            const int kv = (int)(w.h / A.nsub);
            if (A.after_rows && lane == 0) {
                const uint64_t at = (uint64_t)w.k.row0 * A.few_heads + w.h;
                if (w.t0 == 0) A.first_cta[at] = (int)blockIdx.x;
                if (w.t1 == (uint32_t)w.k.nt) A.last_cta[at] = (int)blockIdx.x;
            }
            if (!cr_bar_wait(QEMPTY, qphase ^ 1, &gave_up)) goto out;
            qphase ^= 1;
            if (lane == 0) {
                cr_bar_expect(QFULL, min(16u, A.G) * 128 * cfg::kChunks);
                for (int c = 0; c < cfg::kChunks; ++c)
                    cr_tma_load(sq + c * 16 * 128, &map_q, QFULL, c * 64, (int)(w.h % A.nsub) * 16, kv, w.k.row0);
            }
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                const int key = (int)((w.k.lo / kFewTile + t) * kFewTile + (box << A.box_log2));
                const bool on = lane < boxes * cfg::kChunks && key < w.k.klen;
                const uint32_t bytes = 2 * __popc(__ballot_sync(~0u, on)) * A.box_rows * 128;
                int pg = 0;
                // an ordinary load, as in k_attn_rows
                if (on) pg = A.table[(uint64_t)w.k.kbase * A.max_pages + ((uint32_t)key >> A.page_log2)];
                const int y = key & ((1 << A.page_log2) - 1);
                if (!cr_bar_wait(EMPTY(stage), phase ^ 1, &gave_up)) goto out;
                if (lane == 0) cr_bar_expect(FULL(stage), bytes);
                __syncwarp();
                if (on) {
                    const uint32_t dst = ring + stage * 2 * cfg::kTile + ch * (kFewTile * 128) + ((box << A.box_log2) * 128);
                    cr_tma_load(dst, &map_k, FULL(stage), (int)ch * 64, y, kv, pg);
                    cr_tma_load(dst + cfg::kTile, &map_v, FULL(stage), (int)ch * 64, y, kv, pg);
                }
                if (++stage == cfg::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        if (A.own_list) count_pieces(A.plan, cut, &list);
    } else {
        const uint32_t r4 = lane >> 2, q4 = lane & 3;
        const float c = A.c;
        uint32_t jphase = 0;
        auto meet = [&]() {  // of the four warps
            __syncwarp();
            if (lane == 0) cr_bar_arrive(JOIN);
            const bool ok = cr_bar_wait(JOIN, jphase, &gave_up);
            jphase ^= 1;
            return ok;
        };
        while (w.next()) {
            const uint32_t sub = w.h % A.nsub;
            const uint32_t h0 = w.h / A.nsub * A.G + sub * 16;  // first query head of the rows
            const uint32_t rows = min(16u, A.G - sub * 16);
            uint32_t qa[D / 16][4];
            if (!cr_bar_wait(QFULL, qphase, &gave_up)) goto out;
            qphase ^= 1;
            {
                const uint32_t r = lane & 15;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t u = i * 2 + (lane >> 4);
                    ldsm4<false>(qa[i], sq + (u >> 3) * (16 * 128) + r * 128 + (((u & 7) ^ (r & 7)) << 4));
                    if (!WIDE) qa[i][1] = qa[i][3] = 0;
                }
            }
            __syncwarp();
            if (lane == 0) cr_bar_arrive(QEMPTY);
            float o[D / 8][4];
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
            float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                if (!cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
                const int key = (int)((w.k.lo / kFewTile + t) * kFewTile + warp * 16);  // this warp's first key
                const cr_keys16 see = cr_seen16(key, w.k.lo, w.k.klen);
                if (see.any()) {
                    const uint32_t kt = ring + stage * 2 * cfg::kTile, vt = kt + cfg::kTile;
                    float s[2][4] = {};
                    const uint32_t kr = warp * 16 + (lane & 7) + ((lane >> 4) << 3);
                    const uint32_t vr = warp * 16 + (lane & 15);
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t u = (i * 2 + ((lane >> 3) & 1));
                        uint32_t b[4];
                        ldsm4<false>(b, kt + (u >> 3) * (kFewTile * 128) + kr * 128 + (((u & 7) ^ (kr & 7)) << 4));
                        mma16816<BF16>(s[0], qa[i], b[0], b[1]);
                        mma16816<BF16>(s[1], qa[i], b[2], b[3]);
                    }
                    uint32_t keep[2] = {~0u, ~0u};  // halves of v's registers that are seen
                    if (!see.all()) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                if (!see.sees(i * 8 + (int)q4 * 2 + e)) {
                                    s[i][e] = s[i][2 + e] = -INFINITY;
                                    keep[i] &= e ? 0x0000ffffu : 0xffff0000u;
                                }
                            }
                        }
                    }
                    uint32_t pa[4];
#pragma unroll
                    for (int r = 0; r < (WIDE ? 2 : 1); ++r) {
                        float top = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                        const float m_new = fmaxf(m[r], top);
                        if (__any_sync(~0u, m_new != m[r])) {
                            const float f = m_new == m[r] ? 1.f : cr_exp2((m[r] - m_new) * c);
                            l[r] *= f;
#pragma unroll
                            for (int i = 0; i < D / 8; ++i) {
                                o[i][2 * r] *= f;
                                o[i][2 * r + 1] *= f;
                            }
                            m[r] = m_new;
                        }
                        const float by = fabsf(m[r]) > A.far ? A.c_pow : c;
                        const float off = m[r] == -INFINITY ? 0.f : -m[r] * by;
                        float p[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] = cr_exp2(fmaf(s[i >> 1][2 * r + (i & 1)], by, off));
                        l[r] += (p[0] + p[1]) + (p[2] + p[3]);
                        pa[r] = cr_pack16<BF16>(p[0], p[1]);
                        pa[2 + r] = cr_pack16<BF16>(p[2], p[3]);
                    }
                    if (!WIDE) pa[1] = pa[3] = 0;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t u = i * 2 + (lane >> 4);
                        uint32_t b[4];
                        ldsm4<true>(b, vt + (u >> 3) * (kFewTile * 128) + vr * 128 + (((u & 7) ^ (vr & 7)) << 4));
                        mma16816<BF16>(o[2 * i], pa, b[0] & keep[0], b[1] & keep[1]);
                        mma16816<BF16>(o[2 * i + 1], pa, b[2] & keep[0], b[3] & keep[1]);
                    }
                }
                __syncwarp();
                if (lane == 0) cr_bar_arrive(EMPTY(stage));
                if (++stage == cfg::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            // ---- the four warps' states join: eight rows and 64 columns at a time, four columns a thread ----
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                l[r] += __shfl_xor_sync(~0u, l[r], 1);
                l[r] += __shfl_xor_sync(~0u, l[r], 2);
                if (q4 == 0) join_ml[warp][r4 + 8 * r] = make_float2(m[r] == -INFINITY ? m[r] : m[r] * c, l[r]);
            }
            const int slot = w.slot();
            // a whole block that a shared prefix still joins has a place of its own
            const bool to_own = slot < 0 && w.k.lo > 0;
            const uint64_t place = to_own ? (uint64_t)w.k.row0 * A.few_heads + w.h : (uint64_t)slot;
            float *part = to_own ? A.own : A.part, *part_ml = to_own ? A.own_ml : A.part_ml;
#pragma unroll
            for (int pass = 0; pass < (WIDE ? 2 : 1) * cfg::kChunks; ++pass) {
                const int r = pass / cfg::kChunks, ch = pass % cfg::kChunks;
                if (rows <= 8u * r) break;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<float2 *>(join + (warp * 8 + r4) * 64 + i * 8 + q4 * 2) =
                        make_float2(o[ch * 8 + i][2 * r], o[ch * 8 + i][2 * r + 1]);
                if (!meet()) goto out;
                const uint32_t rr = threadIdx.x >> 4, d4 = ch * 16 + (threadIdx.x & 15), row = 8 * r + rr;
                if (row < rows) {
                    const uint64_t oh = (uint64_t)w.k.row0 * A.q_heads + h0 + row;
                    float mm = -INFINITY, ll = 0.f;
                    for (int v = 0; v < kFewWarps; ++v) mm = fmaxf(mm, join_ml[v][row].x);
                    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int v = 0; v < kFewWarps; ++v) {
                        const float2 ml = join_ml[v][row];
                        const float f = ml.x == -INFINITY ? 0.f : cr_exp2(ml.x - mm);
                        const float4 x = *reinterpret_cast<const float4 *>(join + (v * 8 + rr) * 64 + 4 * (threadIdx.x & 15));
                        ll += ml.y * f;
                        s.x += x.x * f;
                        s.y += x.y * f;
                        s.z += x.z * f;
                        s.w += x.w * f;
                    }
                    if (slot >= 0 || to_own) {
                        reinterpret_cast<float4 *>(part)[(place * (D / 4) + d4) * 16 + row] = s;
                        if (d4 == 0) reinterpret_cast<float2 *>(part_ml)[place * 16 + row] = make_float2(mm, ll);
                    } else {
                        const float inv = ll == 0.f ? 0.f : 1.f / ll;
                        if (4 * d4 < A.head_dim)
                            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.o) + (uint64_t)w.k.row0 * A.o_token +
                                                       (uint64_t)(h0 + row) * A.o_head + 4 * d4) =
                                make_uint2(cr_pack16<BF16>(s.x * inv, s.y * inv), cr_pack16<BF16>(s.z * inv, s.w * inv));
                        if (d4 == 0 && A.lse)
                            A.lse[oh] = (ll == 0.f ? -INFINITY : mm + log2f(ll)) * 0.693147180559945309f;
                    }
                }
                if (!meet()) goto out;
            }
        }
    }
out:
    __syncwarp();
    if (gave_up) {
        if (lane == 0) atomicOr(A.status, CR_FLAG_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
#undef FULL
#undef EMPTY
#undef QFULL
#undef QEMPTY
#undef JOIN
}

// ---- few rows over 8 bits -----------------------------------------------------------------------
// As k_attn_few with half of the bytes.  Numbers are widened to half precision in registers (exact), and the rest of
// a product's arithmetic is arranged so that halves are enough:
//   a head's bfloat16 query is first multiplied by a power of two that brings its largest element to 2^14 .. 2^15
//   (elements 2^28 below it are still exact); scores are 32-bit sums, times that power's inverse and the key block's;
//   weights (at most 2^8, see below) are multiplied by their value block's power over the largest, E, that the warp has
//   met, and by 2^7: they are rounded to 11 bits as long as that is above 2^-14, and are off by less than 2^-31 E
//   otherwise.
// Keys and values are the products' 16-row operand and heads the 8-column one, so that up to eight heads waste nothing
// (scores come out key by head, weights go back in head by key: movmatrix turns them).  The contraction's order is free,
// and so is that of the rows: a lane takes what lies together, for scores D/4 consecutive elements of two keys, for
// values D/8 consecutive elements of four keys, whose bytes it pairs up.
// A head's maximum may lag by 2^8: then a step needs no exchange between lanes but one vote.
// Bound by HBM and latency: 64 contexts to 32,768, 28/4 heads of 128, 89 us (538 MB, 6.0 TB/s) of the call's 141; with
// heads as the 16-row operand and maxima that do not lag the call took 161.  One token over 2,112: 9 to 10 us cold.
// Registers: 114 to 156; WIDE 152 to 168, which at head size 128 leaves 148 (half) or 192 (bfloat16) bytes of spill stores.
template <int D>
struct few8_cfg {
    static constexpr int kTile = kFewTile * D;            // bytes of 64 keys
    static constexpr int kStages = D == 128 ? 6 : 12;
    static constexpr int kQ = 16 * D * 2;
    static constexpr int kJoinRow = 68;                   // floats
    static constexpr int kJoin = kFewWarps * 8 * kJoinRow * 4;
    static constexpr int kSmem = kStages * 2 * kTile + kQ + kJoin + 1024;
};

template <int D, bool BF16, bool WIDE>
__global__ void __launch_bounds__(kFewThreads, 2)
    k_attn_few8(const __grid_constant__ attn_in A, const __grid_constant__ CUtensorMap map_q,
                const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using cfg = few8_cfg<D>;
    constexpr int kDims = D / 4;      // elements of a key that a lane takes
    constexpr int kRun = D / 8;       // elements of a value that a lane takes
    constexpr int kN = WIDE ? 2 : 1;  // groups of eight heads
    extern __shared__ unsigned char dyn[];
    __shared__ __align__(8) unsigned long long bars[2 * cfg::kStages + 3];
    __shared__ __align__(16) float scales[cfg::kStages][16];  // of eight groups of eight keys, and values
    __shared__ float2 join_ml[kFewWarps][16];
    __shared__ int gave_up;
    __shared__ own_list list;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = cr_smem(dyn), ring = (base + 1023u) & ~1023u, sq = ring + cfg::kStages * 2 * cfg::kTile;
    float *join = reinterpret_cast<float *>(dyn + (sq - base) + cfg::kQ);
    const uint32_t bar = cr_smem(bars);
#define FULL(s) (bar + 8u * (s))
#define EMPTY(s) (bar + 8u * (cfg::kStages + (s)))
#define QFULL (bar + 8u * (2 * cfg::kStages))
#define QEMPTY (bar + 8u * (2 * cfg::kStages + 1))
#define JOIN (bar + 8u * (2 * cfg::kStages + 2))

    if (threadIdx.x == 32) {
        cr_tma_prefetch_map(&map_q);
        cr_tma_prefetch_map(&map_k);
        cr_tma_prefetch_map(&map_v);
    }
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int s = 0; s < cfg::kStages; ++s) {
            cr_bar_init(FULL(s), 1 + 16);  // the tile's copies, and those of its scales
            cr_bar_init(EMPTY(s), kFewWarps);
        }
        cr_bar_init(QFULL, 1);
        cr_bar_init(QEMPTY, kFewWarps);
        cr_bar_init(JOIN, kFewWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (uint32_t i = threadIdx.x; i < cfg::kQ / 16; i += kFewThreads)  // rows that no copy writes
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sq + 16 * i), "r"(0));
    cr_fence_async_smem();
    __syncthreads();
    cr_wait_previous();  // as k_attn_few
    cr_launch_next();

    walk w;
    plan_cut cut;
    if (A.own_list) {
        if (warp == kFewWarps) cut = make_list(A.plan, &list, A.status);
        __syncthreads();
        w.begin(list.start, list.blk, A.extra);
    } else {
        w.begin(A.start + blockIdx.x, A.blk, A.extra);
    }
    uint32_t stage = 0, phase = 0, qphase = 0;
    if (warp == kFewWarps) {
        // ---- copies: a lane has one group of eight keys; its scale, and the box that begins there ----
        const uint32_t group = lane & 7;
        while (w.next()) {
            const int kv = (int)(w.h / A.nsub);
            if (A.after_rows && lane == 0) {
                const uint64_t at = (uint64_t)w.k.row0 * A.few_heads + w.h;
                if (w.t0 == 0) A.first_cta[at] = (int)blockIdx.x;
                if (w.t1 == (uint32_t)w.k.nt) A.last_cta[at] = (int)blockIdx.x;
            }
            if (!cr_bar_wait(QEMPTY, qphase ^ 1, &gave_up)) goto out;
            qphase ^= 1;
            if (lane == 0) {
                cr_bar_expect(QFULL, min(16u, A.G) * 128 * (D / 64));
                for (int c = 0; c < D / 64; ++c)
                    cr_tma_load(sq + c * 16 * 128, &map_q, QFULL, c * 64, (int)(w.h % A.nsub) * 16, kv, w.k.row0);
            }
            const int32_t *row = A.table + (uint64_t)w.k.kbase * A.max_pages;
            const uint32_t tile0 = (uint32_t)w.k.lo / kFewTile;
            // behind the sequence's end: ~0; n_pages stands for what is no page, whose copy is of zeros
            auto page_of = [&](uint32_t t) {
                const uint32_t at = (tile0 + t) * kFewTile + group * 8;
                return t < w.t1 && (int)at < w.k.klen ? min((uint32_t)row[at >> A.page_log2], A.n_pages) : ~0u;
            };
            uint32_t next = page_of(w.t0);
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                const uint32_t in_page = ((tile0 + t) * kFewTile + group * 8) & ((1u << A.page_log2) - 1);
                const uint32_t page = next;
                next = page_of(t + 1);  // on its way while this tile waits for its place
                const bool on = page < A.n_pages, brings = lane < 8 && page != ~0u && (group * 8 & (A.box_rows - 1)) == 0;
                const uint32_t bytes = 2 * __popc(__ballot_sync(~0u, brings)) * A.box_rows * D;
                const uint64_t scale = on ? (((uint64_t)page * A.kv_heads + kv) << A.nb_log2) + (in_page >> A.block_log2) : 0;
                if (!cr_bar_wait(EMPTY(stage), phase ^ 1, &gave_up)) goto out;
                if (lane == 0) cr_bar_expect(FULL(stage), bytes);
                __syncwarp();
                if (brings) {
                    const uint32_t dst = ring + stage * 2 * cfg::kTile + group * 8 * D;
                    cr_tma_load(dst, &map_k, FULL(stage), 0, (int)in_page, kv, (int)page);
                    cr_tma_load(dst + cfg::kTile, &map_v, FULL(stage), 0, (int)in_page, kv, (int)page);
                }
                if (lane < 16) cr_copy_word(cr_smem(&scales[stage][lane]), (lane < 8 ? A.k_scale : A.v_scale) + scale, on, FULL(stage));
                if (++stage == cfg::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        if (A.own_list) count_pieces(A.plan, cut, &list);
    } else {
        const uint32_t r4 = lane >> 2, q4 = lane & 3;
        uint32_t jphase = 0;
        auto meet = [&]() {  // of the four warps
            __syncwarp();
            if (lane == 0) cr_bar_arrive(JOIN);
            const bool ok = cr_bar_wait(JOIN, jphase, &gave_up);
            jphase ^= 1;
            return ok;
        };
        while (w.next()) {
            const uint32_t sub = w.h % A.nsub;
            const uint32_t h0 = w.h / A.nsub * A.G + sub * 16;  // first query head of the rows
            const uint32_t rows = min(16u, A.G - sub * 16);
            uint32_t qb[kN][D / 16][2];  // head 8 n + r4
            float cs[kN][2];             // what makes scores of sums: heads 8 n + 2 q4 and the next
            if (!cr_bar_wait(QFULL, qphase, &gave_up)) goto out;
            qphase ^= 1;
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                const uint32_t row = r4 + 8 * n;
                uint32_t x[kDims / 2];
#pragma unroll
                for (int k = 0; k < kDims / 8; ++k) {
                    const uint32_t u = q4 * (kDims / 8) + k;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(x[4 * k]), "=r"(x[4 * k + 1]), "=r"(x[4 * k + 2]), "=r"(x[4 * k + 3])
                                 : "r"(sq + (u >> 3) * (16 * 128) + row * 128 + (((u & 7) ^ (row & 7)) << 4)));
                }
                float c = A.c;
                if (BF16) {
                    uint32_t top = 0;  // the largest magnitude's bits
#pragma unroll
                    for (int k = 0; k < kDims / 2; ++k) top = max(top, max(x[k] << 16 & 0x7fffffffu, x[k] & 0x7fff0000u));
                    top = max(top, __shfl_xor_sync(~0u, top, 1));
                    top = max(top, __shfl_xor_sync(~0u, top, 2));
                    const int up = max(-113, min(113, 14 + 127 - (int)(top >> 23)));
                    const float f = __uint_as_float((uint32_t)(127 + up) << 23);
                    c *= __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
                    for (int k = 0; k < kDims / 2; ++k)
                        x[k] = cr_pack16<false>(__uint_as_float(x[k] << 16) * f, __uint_as_float(x[k] & 0xffff0000u) * f);
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    qb[n][i][0] = x[2 * i];
                    qb[n][i][1] = x[2 * i + 1];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) cs[n][e] = __shfl_sync(~0u, c, (2 * q4 + e) * 4);
            }
            __syncwarp();
            if (lane == 0) cr_bar_arrive(QEMPTY);
            // o[n][t]: elements r4 kRun + 2 t (0, 1) and the next (2, 3) of heads 8 n + 2 q4 (0, 2) and the next (1, 3),
            // in units of 2^-7 E
            float o[kN][D / 16][4];
            float m[kN][2], l[kN][2];
#pragma unroll
            for (int n = 0; n < kN; ++n) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
                // the lowest finite number: a score is that or above it by more than may be, and one that is not seen,
                // minus infinity, has weight 0 beside it
                m[n][0] = m[n][1] = -0x1.fffffep127f;
                l[n][0] = l[n][1] = 0.f;
            }
            float E = 0.f, per_E = 0.f;  // per_E: 2^7 / E
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                if (!cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
                const int key = (int)((w.k.lo / kFewTile + t) * kFewTile + warp * 16);  // this warp's first key
                const cr_keys16 see = cr_seen16(key, w.k.lo, w.k.klen);
                if (see.any()) {
                    const uint32_t kt = ring + stage * 2 * cfg::kTile, vt = kt + cfg::kTile;
                    const float2 ks = *reinterpret_cast<const float2 *>(&scales[stage][2 * warp]);
                    const float2 vs = *reinterpret_cast<const float2 *>(&scales[stage][8 + 2 * warp]);
                    // keys warp 16 + r4 and 8 more
                    uint32_t c4[2][kDims / 4];
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const uint32_t kr = warp * 16 + g * 8 + r4, turn = D == 128 ? kr & 7 : (kr >> 1) & 3;
#pragma unroll
                        for (int k = 0; k < kDims / 16; ++k)
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(c4[g][4 * k]), "=r"(c4[g][4 * k + 1]), "=r"(c4[g][4 * k + 2]), "=r"(c4[g][4 * k + 3])
                                         : "r"(kt + kr * D + (((q4 * (kDims / 16) + k) ^ turn) << 4)));
                    }
                    // four keys' runs; words of four elements
                    uint32_t v[4][kRun / 4];
                    auto load_values = [&]() {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t vr = warp * 16 + (e >> 1) * 8 + 2 * q4 + (e & 1);
                            if (D == 128) {
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                             : "=r"(v[e][0]), "=r"(v[e][1]), "=r"(v[e][kRun / 4 - 2]), "=r"(v[e][kRun / 4 - 1])
                                             : "r"(vt + vr * D + ((r4 ^ (vr & 7)) << 4)));
                            } else {
                                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];"
                                             : "=r"(v[e][0]), "=r"(v[e][1])
                                             : "r"(vt + vr * D + (((r4 >> 1) ^ ((vr >> 1) & 3)) << 4) + (r4 & 1) * 8));
                            }
                        }
                    };
                    if (!WIDE) load_values();  // sixteen heads leave no registers for them yet
                    float s[kN][2][4] = {};  // two sums, so that a product does not wait for the one before
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        uint32_t a[4];
                        cr_e4m3_halves(c4[0][i], a[0], a[2]);
                        cr_e4m3_halves(c4[1][i], a[1], a[3]);
#pragma unroll
                        for (int n = 0; n < kN; ++n) mma16816<false>(s[n][i & 1], a, qb[n][i][0], qb[n][i][1]);
                    }
                    float x[kN][4];  // base-2 logarithms
                    bool over = false;
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[n][e] = (s[n][0][e] + s[n][1][e]) * (cs[n][e & 1] * (e < 2 ? ks.x : ks.y));
                    if (!see.all()) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!see.sees((e >> 1) * 8 + (int)r4))
#pragma unroll
                                for (int n = 0; n < kN; ++n) x[n][e] = -INFINITY;
                    }
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) over |= x[n][e] - m[n][e & 1] > 8.f;
                    const float most = fmaxf(vs.x, vs.y);
                    if (__any_sync(~0u, over) || most > E) {
                        float grown = 1.f;  // of E
                        if (most > E) {
                            grown = E / most;
                            E = most;
                            per_E = 128.f / E;
                        }
#pragma unroll
                        for (int n = 0; n < kN; ++n) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float top = fmaxf(x[n][e], x[n][2 + e]);
                                top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
                                top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
                                top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
                                const float m_new = fmaxf(m[n][e], top);
                                float r = m_new == m[n][e] ? 1.f : cr_exp2(m[n][e] - m_new);
                                m[n][e] = m_new;
                                l[n][e] *= r;
                                r *= grown;
#pragma unroll
                                for (int i = 0; i < D / 16; ++i) {
                                    o[n][i][e] *= r;
                                    o[n][i][2 + e] *= r;
                                }
                            }
                        }
                    }
                    const float by[2] = {vs.x * per_E, vs.y * per_E};
                    uint32_t pb[kN][2];
#pragma unroll
                    for (int n = 0; n < kN; ++n) {
                        float p[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e] = cr_exp2(x[n][e] - m[n][e & 1]);
                        l[n][0] += p[0] + p[2];
                        l[n][1] += p[1] + p[3];
#pragma unroll
                        for (int g = 0; g < 2; ++g)
                            asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;"
                                         : "=r"(pb[n][g])
                                         : "r"(cr_pack16<false>(p[2 * g] * by[g], p[2 * g + 1] * by[g])));
                    }
                    if (WIDE) load_values();
                    if (!see.all()) {  // what is not seen may be no number
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!see.sees((e >> 1) * 8 + (int)q4 * 2 + (e & 1)))
#pragma unroll
                                for (int i = 0; i < kRun / 4; ++i) v[e][i] = 0;
                    }
#pragma unroll
                    for (int i = 0; i < kRun / 4; ++i) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {  // elements 4 i + 2 h and the next: bytes of two keys side by side
                            const uint32_t lo = __byte_perm(v[0][i], v[1][i], h ? 0x7362 : 0x5140);
                            const uint32_t hi = __byte_perm(v[2][i], v[3][i], h ? 0x7362 : 0x5140);
                            uint32_t a[4];
                            cr_e4m3_halves(lo, a[0], a[1]);
                            cr_e4m3_halves(hi, a[2], a[3]);
#pragma unroll
                            for (int n = 0; n < kN; ++n) mma16816<false>(o[n][2 * i + h], a, pb[n][0], pb[n][1]);
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) cr_bar_arrive(EMPTY(stage));
                if (++stage == cfg::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            // ---- the four warps' states join: eight heads and 64 columns at a time, four columns a thread ----
            const float unit = E * 0x1p-7f;
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = l[n][e];
                    x += __shfl_xor_sync(~0u, x, 4);
                    x += __shfl_xor_sync(~0u, x, 8);
                    x += __shfl_xor_sync(~0u, x, 16);
                    if (r4 == 0) join_ml[warp][8 * n + 2 * q4 + e] = make_float2(x == 0.f ? -INFINITY : m[n][e], x);
                }
            const int slot = w.slot();
            // a whole block that a shared prefix still joins has a place of its own
            const bool to_own = slot < 0 && w.k.lo > 0;
            const uint64_t place = to_own ? (uint64_t)w.k.row0 * A.few_heads + w.h : (uint64_t)slot;
            float *part = to_own ? A.own : A.part, *part_ml = to_own ? A.own_ml : A.part_ml;
#pragma unroll
            for (int pass = 0; pass < kN * (D / 64); ++pass) {
                const int n = pass / (D / 64), ch = pass % (D / 64);
                if (rows <= 8u * n) break;
                // column 8 r + i: element r kRun + ch * 8 + i
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float *to = join + (warp * 8 + 2 * q4 + e) * cfg::kJoinRow + r4 * 8;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        *reinterpret_cast<float4 *>(to + 4 * i) =
                            make_float4(o[n][ch * 4 + 2 * i][e] * unit, o[n][ch * 4 + 2 * i][2 + e] * unit,
                                        o[n][ch * 4 + 2 * i + 1][e] * unit, o[n][ch * 4 + 2 * i + 1][2 + e] * unit);
                }
                if (!meet()) goto out;
                const uint32_t rr = threadIdx.x >> 4, col = threadIdx.x & 15, row = 8 * n + rr;
                const uint32_t d4 = ((col >> 1) * kRun + ch * 8 + (col & 1) * 4) / 4;
                if (row < rows) {
                    const uint64_t oh = (uint64_t)w.k.row0 * A.q_heads + h0 + row;
                    float mm = -INFINITY, ll = 0.f;
                    for (int v = 0; v < kFewWarps; ++v) mm = fmaxf(mm, join_ml[v][row].x);
                    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int v = 0; v < kFewWarps; ++v) {
                        const float2 ml = join_ml[v][row];
                        const float f = ml.x == -INFINITY ? 0.f : cr_exp2(ml.x - mm);
                        const float4 x = *reinterpret_cast<const float4 *>(join + (v * 8 + rr) * cfg::kJoinRow + 4 * col);
                        ll += ml.y * f;
                        s.x += x.x * f;
                        s.y += x.y * f;
                        s.z += x.z * f;
                        s.w += x.w * f;
                    }
                    if (slot >= 0 || to_own) {
                        reinterpret_cast<float4 *>(part)[(place * (D / 4) + d4) * 16 + row] = s;
                        if (d4 == 0) reinterpret_cast<float2 *>(part_ml)[place * 16 + row] = make_float2(mm, ll);
                    } else {
                        const float inv = ll == 0.f ? 0.f : 1.f / ll;
                        if (4 * d4 < A.head_dim)
                            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.o) + (uint64_t)w.k.row0 * A.o_token +
                                                       (uint64_t)(h0 + row) * A.o_head + 4 * d4) =
                                make_uint2(cr_pack16<BF16>(s.x * inv, s.y * inv), cr_pack16<BF16>(s.z * inv, s.w * inv));
                        if (d4 == 0 && A.lse)
                            A.lse[oh] = (ll == 0.f ? -INFINITY : mm + log2f(ll)) * 0.693147180559945309f;
                    }
                }
                if (!meet()) goto out;
            }
        }
    }
out:
    __syncwarp();
    if (gave_up) {
        if (lane == 0) atomicOr(A.status, CR_FLAG_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
#undef FULL
#undef EMPTY
#undef QFULL
#undef QEMPTY
#undef JOIN
}

// ---- host -------------------------------------------------------------------------------------
typedef CUresult (*encode_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

encode_fn encoder()
{
    static encode_fn fn = [] {
        cudaDriverEntryPointQueryResult q;
        void *p = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<encode_fn>(p);
    }();
    return fn;
}

// A 4-D map of 16-bit elements: dims and strides (elements) from the second dimension on, boxes of
// 64 elements of the first.  bytes != 0: of 8-bit elements, so many in a box.
int encode_map(cr_ctx *ctx, CUtensorMap *map, bool bf16, const void *base, const uint64_t dim[4], const uint64_t stride[3],
               const uint32_t box[3], bool stream_once, uint32_t bytes = 0)
{
    encode_fn fn = encoder();
    if (!fn) return cr_fail(ctx, CR_ECUDA, "cuTensorMapEncodeTiled is not available from this driver");
    cuuint64_t st[3];
    for (int i = 0; i < 3; ++i) st[i] = dim[i + 1] == 1 ? 16 : stride[i] * (bytes ? 1 : 2);  // 1: never stepped over
    const cuuint32_t bx[4] = {bytes ? bytes : 64, box[0], box[1], box[2]}, es[4] = {1, 1, 1, 1};
    const cuuint64_t dm[4] = {dim[0], dim[1], dim[2], dim[3]};
    const CUtensorMapDataType type = bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                           : (bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16);
    const CUresult r = fn(map, type, 4, const_cast<void *>(base), dm, st, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                          stream_once ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cr_fail(ctx, CR_EINVAL, "tensor map rejected (%d): check pointers and strides", (int)r);
    return CR_OK;
}

// Keys and values of a call.
struct kv_desc {
    bool paged, bf16, e4m3;
    uint32_t heads, dim;
    const void *k, *v;
    uint64_t k_row, k_head, v_row, v_head;  // elements between tokens, heads
    // packed
    uint32_t n_kv;
    const int32_t *cu_k;
    // paged
    const cr_kv_pages *pg;
    const float *k_scale, *v_scale;  // 8 bits
};

int kv_map(cr_ctx *ctx, CUtensorMap *map, const kv_desc &K, bool value, uint32_t box_rows)
{
    uint64_t dim[4] = {K.dim, 0, K.heads, 1}, st[3] = {value ? K.v_row : K.k_row, value ? K.v_head : K.k_head, 8};
    if (K.paged) {
        dim[1] = K.pg->page;
        dim[3] = K.pg->n_pages;
        st[2] = K.pg->page_stride;
    } else if (K.n_kv) {
        dim[1] = K.n_kv;
    } else {
        dim[1] = dim[2] = 1;  // one row stands for no keys at all (cr_attn_packed)
    }
    const uint32_t box[3] = {box_rows, 1, 1};
    return encode_map(ctx, map, K.bf16, value ? K.v : K.k, dim, st, box, K.paged, K.e4m3 ? (K.dim <= 64 ? 64 : 128) : 0);
}

uint32_t ilog2(uint32_t v)
{
    uint32_t b = 0;
    while ((2u << b) <= v) ++b;
    return b;
}

// Scratch of one list of work.
struct plan_mem {
    size_t bytes;
    size_t blk, cum, start, joins, ctas, first, of_token;
    uint64_t n_marks;
    // tokens: of groups; marks: (token, head) places of first_cta and last_cta
    plan_mem(uint32_t max_blk, uint32_t max_cta, uint32_t n, uint32_t tokens, uint64_t marks)
    {
        bytes = 0;
        n_marks = marks;
        auto take = [&](size_t b) {
            const size_t at = bytes;
            bytes += (b + 255) & ~(size_t)255;
            return at;
        };
        blk = take(sizeof(attn_blk) * ((size_t)max_blk + 1));
        cum = take(max_blk > kPlanShared ? 8 * ((size_t)max_blk + 2) : 0);
        start = take(sizeof(attn_start) * ((size_t)max_cta + 2));
        joins = take(4 * ((size_t)max_cta + 2));
        ctas = take(8 * (size_t)marks);
        first = take(n > kPlanShared ? 4 * ((size_t)n + 1) : 0);
        of_token = take(4 * (size_t)tokens);
    }
    void point(char *base, plan_in &p, attn_in &a) const
    {
        p.blk = reinterpret_cast<attn_blk *>(base + blk);
        p.cum = reinterpret_cast<unsigned long long *>(base + cum);
        p.start = reinterpret_cast<attn_start *>(base + start);
        p.first = reinterpret_cast<uint32_t *>(base + first);
        a.blk = p.blk;
        p.joins = reinterpret_cast<uint32_t *>(base + joins);
        a.joins = p.joins;
        a.first_cta = reinterpret_cast<int32_t *>(base + ctas);
        a.last_cta = a.first_cta + n_marks;
        p.of_token = reinterpret_cast<int32_t *>(base + of_token);
        a.start = p.start;
        a.extra = p.extra;
        a.ncta = p.max_cta;
        a.of_token = p.of_token;
    }
};

bool aligned(const void *p, uint64_t a, uint64_t b) { return ((uintptr_t)p & 15) == 0 && (a & 7) == 0 && (b & 7) == 0; }

int check_heads(cr_ctx *ctx, const char *who, const cr_attn_args *a, uint32_t dtype, uint32_t kv_heads, uint32_t dim)
{
    if (dtype > CR_DTYPE_FP16) return cr_fail(ctx, CR_EINVAL, "%s: dtype %u", who, dtype);
    if (kv_heads == 0 || kv_heads > 4096 || a->q_heads == 0 || a->q_heads % kv_heads || a->q_heads / kv_heads > 128)
        return cr_fail(ctx, CR_EINVAL, "%s: %u query heads on %u key heads", who, a->q_heads, kv_heads);
    if (dim == 0 || dim > 128 || (dim & 7)) return cr_fail(ctx, CR_EINVAL, "%s: head_dim %u", who, dim);
    if (!(a->scale > 0.f) || isinf(a->scale)) return cr_fail(ctx, CR_EINVAL, "%s: scale must be finite and positive", who);
    if (a->reserved) return cr_fail(ctx, CR_EINVAL, "%s: reserved must be 0", who);
    if (a->n > (1u << 24) || a->n_tokens > (1u << 30)) return cr_fail(ctx, CR_EINVAL, "%s: too many entries or tokens", who);
    if (a->n_tokens && (!a->d_q || !a->d_o)) return cr_fail(ctx, CR_EINVAL, "%s: NULL pointer", who);
    if (!aligned(a->d_q, a->q_token, a->q_head) || !aligned(a->d_o, a->o_token, a->o_head))
        return cr_fail(ctx, CR_EINVAL, "%s: queries and outputs must be 16-byte aligned, strides multiples of 8", who);
    return CR_OK;
}

void fill_common(attn_in &A, cr_ctx *ctx, const cr_attn_args *a, const kv_desc &K)
{
    A.paged = K.paged;
    A.G = a->q_heads / K.heads;
    A.nsub = 1;
    A.tq = kRowsTile / A.G;
    A.q_heads = a->q_heads;
    A.kv_heads = K.heads;
    A.head_dim = K.dim;
    A.c = fminf(a->scale * 1.44269504088896341f, 0x1.fffffep127f);
    A.c_pow = coarse(A.c);
    A.c_rest = A.c / A.c_pow;
    A.far = kFar / A.c;
    A.causal = a->causal != 0;
    A.o = a->d_o;
    A.o_token = a->o_token;
    A.o_head = a->o_head;
    A.o_wide = !((uintptr_t)a->d_o & 31) && !((a->o_token | a->o_head) & 15);
    A.lse = a->d_lse;
    A.status = ctx->d_status;
    if (K.paged) {
        A.table = K.pg->d_table;
        A.max_pages = K.pg->max_pages;
        A.page_log2 = ilog2(K.pg->page);
        A.n_pages = K.pg->n_pages;
        A.k_scale = K.k_scale;
        A.v_scale = K.v_scale;
        if (K.e4m3) {
            A.block_log2 = ilog2(K.pg->block);
            A.nb_log2 = A.page_log2 - A.block_log2;
        }
    }
}

// Raises a kernel's limit of dynamic shared memory, once per device (bits of `done`).
template <typename K>
int raise_smem(cr_ctx *ctx, K kern, int bytes, unsigned long long &done)
{
    const unsigned long long bit = 1ull << (ctx->device & 63);
    if (done & bit) return CR_OK;
    CR_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    done |= bit;
    return CR_OK;
}

int query_map(cr_ctx *ctx, CUtensorMap *map, const attn_in &A, const kv_desc &K, const cr_attn_args *a, uint32_t heads,
              uint32_t tokens)
{
    const uint64_t dim[4] = {K.dim, A.G, K.heads, a->n_tokens}, st[3] = {a->q_head, a->q_head * A.G, a->q_token};
    const uint32_t box[3] = {heads, 1, tokens};
    return encode_map(ctx, map, K.bf16, a->d_q, dim, st, box, false);
}

template <int D, bool BF16, bool E8>
int launch_rows(cr_ctx *ctx, const attn_in &A, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    CUtensorMap mq, mk, mv;
    CR_TRY(query_map(ctx, &mq, A, K, a, A.G, A.tq));
    CR_TRY(kv_map(ctx, &mk, K, false, A.box_rows));
    CR_TRY(kv_map(ctx, &mv, K, true, A.box_rows));
    auto kern = k_attn_rows<D, BF16, E8>;
    static unsigned long long raised = 0;
    CR_TRY(raise_smem(ctx, kern, rows_cfg<D, E8>::kSmem, raised));
    CR_TRY(cr_launch_early(ctx, "k_attn_rows", kern, dim3(ctas), rows_threads(E8), rows_cfg<D, E8>::kSmem, A, mq, mk, mv));
    if (ctas > 1 && !A.to_pfx)
        CR_TRY(cr_launch_early(ctx, "k_attn_join", k_attn_join<D, BF16, 2 * kRowsTile>, dim3(4 * ctx->num_sms), 256, 0, A));
    return CR_OK;
}

template <bool E8>
int rows_of(cr_ctx *ctx, const attn_in &A, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    if (K.dim <= 64) return K.bf16 ? launch_rows<64, true, E8>(ctx, A, K, a, ctas) : launch_rows<64, false, E8>(ctx, A, K, a, ctas);
    return K.bf16 ? launch_rows<128, true, E8>(ctx, A, K, a, ctas) : launch_rows<128, false, E8>(ctx, A, K, a, ctas);
}
int rows(cr_ctx *ctx, const attn_in &A, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    return K.e4m3 ? rows_of<true>(ctx, A, K, a, ctas) : rows_of<false>(ctx, A, K, a, ctas);
}

template <int D, bool BF16, bool WIDE, bool E8>
int launch_few(cr_ctx *ctx, const attn_in &A, const attn_in *R, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    CUtensorMap mq, mk, mv;
    CR_TRY(query_map(ctx, &mq, A, K, a, A.G < 16 ? A.G : 16, 1));
    CR_TRY(kv_map(ctx, &mk, K, false, A.box_rows));
    CR_TRY(kv_map(ctx, &mv, K, true, A.box_rows));
    auto kern = k_attn_few<D, BF16, WIDE>;
    int smem = few_cfg<D>::kSmem;
    if (E8) {
        kern = k_attn_few8<D, BF16, WIDE>;
        smem = few8_cfg<D>::kSmem;
    }
    static unsigned long long raised = 0;
    CR_TRY(raise_smem(ctx, kern, smem, raised));
    CR_TRY(cr_launch_early(ctx, "k_attn_few", kern, dim3(ctas), kFewThreads, smem, A, mq, mk, mv));
    if (R)
        CR_TRY(cr_launch_early(ctx, "k_attn_decode_join", k_attn_decode_join<D, BF16>, dim3(a->n, A.few_heads), 256, 0, A, *R));
    else if (ctas > 1)
        CR_TRY(cr_launch_early(ctx, "k_attn_join", k_attn_join<D, BF16, 16>, dim3(min(ctas - 1, 2 * (uint32_t)ctx->num_sms)), 256, 0, A));
    return CR_OK;
}

template <int D, bool BF16>
int few_of(cr_ctx *ctx, const attn_in &A, const attn_in *R, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    const bool wide = A.G > 8;
    if (K.e4m3)
        return wide ? launch_few<D, BF16, true, true>(ctx, A, R, K, a, ctas) : launch_few<D, BF16, false, true>(ctx, A, R, K, a, ctas);
    return wide ? launch_few<D, BF16, true, false>(ctx, A, R, K, a, ctas) : launch_few<D, BF16, false, false>(ctx, A, R, K, a, ctas);
}
int few(cr_ctx *ctx, const attn_in &A, const attn_in *R, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    if (K.dim <= 64) return K.bf16 ? few_of<64, true>(ctx, A, R, K, a, ctas) : few_of<64, false>(ctx, A, R, K, a, ctas);
    return K.bf16 ? few_of<128, true>(ctx, A, R, K, a, ctas) : few_of<128, false>(ctx, A, R, K, a, ctas);
}

// The list of work of a call, and that of its groups.  A short list for few CTAs is made by fewer threads, whose
// barriers are cheaper (one prompt of 512 tokens: 7,600 cycles with 512 threads, 6,400 with 256).
template <int KIND>
int launch_plan(cr_ctx *ctx, const plan_in &a, const plan_in *b)
{
    if (a.n <= 256 && a.max_blk <= 256 && a.max_cta < 256)
        return cr_launch_early(ctx, "k_attn_plan", k_attn_plan<KIND, 256>, dim3(b ? 2 : 1), 256, 0, a, b ? *b : a, ctx->d_status);
    return cr_launch_early(ctx, "k_attn_plan", k_attn_plan<KIND, 512>, dim3(b ? 2 : 1), 512, 0, a, b ? *b : a, ctx->d_status);
}

// Pieces of a list of work: two per CTA at most.
int part_mem(cr_ctx *ctx, int slot, attn_in &A, uint32_t ctas, uint32_t rows_per_piece, uint32_t D)
{
    const size_t n = 2 * (size_t)ctas * rows_per_piece;
    void *p;
    CR_TRY(cr_scratch(ctx, slot, n * (D + 2) * 4, &p));
    A.part = static_cast<float *>(p);
    A.part_ml = A.part + n * D;
    return CR_OK;
}

// Two tiles a CTA at least (64 tokens over 2,048 cached: 24.4 us a call with four, 20.9 with two); a piece costs about
// as much as three tiles of 128 keys, or six of 64.
constexpr uint32_t kRowsMinTiles = 2, kFewMinTiles = 2, kRowsPieceCost = 3, kFewPieceCost = 6, kFewPieceCost8 = 8;

constexpr uint64_t kAloneTiles = 8192;

int attn_many(cr_ctx *ctx, const cr_attn_args *a, const kv_desc &K)
{
    if (a->n_tokens == 0 || a->n == 0) return CR_OK;
    attn_in A = {};
    fill_common(A, ctx, a, K);
    A.box_rows = K.paged && K.pg->page < kRowsTile ? K.pg->page : kRowsTile;
    A.box_log2 = ilog2(A.box_rows);
    plan_in p = {};
    p.cu_q = a->d_cu_q;
    p.cu_k = K.cu_k;
    p.seqs = a->d_seqs;
    p.n = a->n;
    p.n_tokens = a->n_tokens;
    p.n_kv = K.n_kv;
    p.heads = K.heads;
    p.causal = A.causal;
    p.tok_blk = 2 * A.tq;
    p.max_blk = a->n_tokens / p.tok_blk + (a->n < a->n_tokens ? a->n : a->n_tokens);
    p.min_tiles = kRowsMinTiles;
    p.piece_cost = kRowsPieceCost;
    p.extra = kExtra;
    if (K.paged) {
        p.lens = K.pg->d_lens;
        p.n_seqs = K.pg->n_seqs;
        p.max_len = K.pg->max_pages * K.pg->page;
    }
    p.max_cta = min((uint32_t)ctx->num_sms, kMaxCtas);
    const plan_mem mem(p.max_blk, p.max_cta, a->n, 0, 0);
    void *base;
    CR_TRY(cr_scratch(ctx, SCR_ATTN_PLAN, mem.bytes, &base));
    mem.point(static_cast<char *>(base), p, A);
    CR_TRY(part_mem(ctx, SCR_ATTN_PART, A, p.max_cta, 2 * kRowsTile, K.dim <= 64 ? 64 : 128));
    if (K.paged)
        CR_TRY(launch_plan<PLAN_PAGED>(ctx, p, nullptr));
    else
        CR_TRY(launch_plan<PLAN_PACKED>(ctx, p, nullptr));
    return rows(ctx, A, K, a, p.max_cta);
}

}  // namespace

static int paged_desc(cr_ctx *ctx, const char *who, const cr_kv_pages *pg, uint32_t layer, kv_desc &K)
{
    CR_TRY(cr_pages_check(ctx, who, pg));
    if (layer >= pg->layers) return cr_fail(ctx, CR_EINVAL, "%s: layer %u of %u", who, layer, pg->layers);
    K = kv_desc{};
    K.paged = true;
    K.bf16 = cr_is_bf16(pg->dtype);
    K.e4m3 = cr_in_8bit(pg->dtype);
    K.heads = pg->kv_heads;
    K.dim = pg->head_dim;
    K.k = static_cast<const uint8_t *>(pg->d_cache) + (K.e4m3 ? 1 : 2) * (layer * pg->layer_stride);
    K.v = static_cast<const uint8_t *>(K.k) + (K.e4m3 ? 1 : 2) * pg->kv_stride;
    if (K.e4m3) {
        const uint64_t plane = ((uint64_t)pg->n_pages * pg->kv_heads) * (pg->page / pg->block);
        K.k_scale = pg->d_scale + 2 * layer * plane;
        K.v_scale = K.k_scale + plane;
    }
    K.k_row = K.v_row = pg->token_stride;
    K.k_head = K.v_head = pg->head_stride;
    K.pg = pg;
    return CR_OK;
}

extern "C" int cr_attn_packed(cr_ctx *ctx, const cr_attn_args *args, uint32_t dtype, uint32_t kv_heads, uint32_t head_dim,
                              const void *d_k, uint64_t k_token, uint64_t k_head, const void *d_v, uint64_t v_token,
                              uint64_t v_head, const int32_t *d_cu_k, uint32_t n_kv)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_attn_packed");
    if (!args) return cr_fail(ctx, CR_EINVAL, "cr_attn_packed: args is NULL");
    CR_TRY(check_heads(ctx, "cr_attn_packed", args, dtype, kv_heads, head_dim));
    if (args->n && !args->d_cu_q) return cr_fail(ctx, CR_EINVAL, "cr_attn_packed: d_cu_q is NULL");
    if (n_kv > (1u << 30) || (n_kv && (!d_k || !d_v)) || !aligned(d_k, k_token, k_head) || !aligned(d_v, v_token, v_head))
        return cr_fail(ctx, CR_EINVAL, "cr_attn_packed: keys and values must be 16-byte aligned, strides multiples of 8");
    kv_desc K = {};
    K.bf16 = dtype == CR_DTYPE_BF16;
    K.heads = kv_heads;
    K.dim = head_dim;
    K.k = d_k;
    K.v = d_v;
    K.k_row = k_token;
    K.k_head = k_head;
    K.v_row = v_token;
    K.v_head = v_head;
    K.n_kv = n_kv;
    K.cu_k = d_cu_k ? d_cu_k : args->d_cu_q;
    if (n_kv == 0) K.k = K.v = args->d_q;  // nothing to map: a query's row is copied, which no query sees
    return attn_many(ctx, args, K);
}

extern "C" int cr_attn_paged(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, const cr_attn_args *args)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_attn_paged");
    if (!args) return cr_fail(ctx, CR_EINVAL, "cr_attn_paged: args is NULL");
    kv_desc K;
    CR_TRY(paged_desc(ctx, "cr_attn_paged", pages, layer, K));
    CR_TRY(check_heads(ctx, "cr_attn_paged", args, cr_is_bf16(pages->dtype) ? CR_DTYPE_BF16 : CR_DTYPE_FP16, pages->kv_heads, pages->head_dim));
    if (args->n && !args->d_cu_q) return cr_fail(ctx, CR_EINVAL, "cr_attn_paged: d_cu_q is NULL");
    return attn_many(ctx, args, K);
}

extern "C" int cr_attn_decode(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, const cr_attn_args *args,
                              const int32_t *d_group_off, const int32_t *d_shared, uint32_t n_groups)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_attn_decode");
    if (!args) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: args is NULL");
    kv_desc K;
    CR_TRY(paged_desc(ctx, "cr_attn_decode", pages, layer, K));
    CR_TRY(check_heads(ctx, "cr_attn_decode", args, cr_is_bf16(pages->dtype) ? CR_DTYPE_BF16 : CR_DTYPE_FP16, pages->kv_heads, pages->head_dim));
    if (args->n_tokens != args->n) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: one query token per entry");
    if (n_groups && (!d_group_off || !d_shared)) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: NULL groups");
    if (n_groups > (1u << 24)) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: %u groups", n_groups);
    if (args->n == 0) return CR_OK;
    if (args->n == 1) n_groups = 0;  // nobody to share with
    // 8 bits: where the rows cannot hold much, every sequence reads its prefix itself, which saves two kernels.  Both take
    // equally long at about 8,300 tiles of 64 keys and a key head, whatever they are made of (heads of 64 and 128, 2 and
    // 8 key heads, 4 to 128 sequences: 13 to 20 us so and 25 to 37 in groups at 4,000 tiles and fewer; at 33,000 83 to 100
    // and 34 to 50).
    if (K.e4m3 && (uint64_t)args->n * K.heads * cr_key_tiles((int)(pages->max_pages * pages->page), kFewTile) <= kAloneTiles) n_groups = 0;

    const uint32_t D = K.dim <= 64 ? 64 : 128;
    attn_in F = {}, R = {};
    fill_common(F, ctx, args, K);
    F.nsub = (F.G + 15) / 16;
    F.causal = 0;
    R = F;
    R.nsub = 1;
    F.box_rows = pages->page < kFewTile ? pages->page : kFewTile;
    F.box_log2 = ilog2(F.box_rows);
    R.box_rows = pages->page < kRowsTile ? pages->page : kRowsTile;
    R.box_log2 = ilog2(R.box_rows);

    plan_in f = {};
    f.seqs = args->d_seqs;
    f.lens = pages->d_lens;
    f.goff = d_group_off;
    f.shared = d_shared;
    f.n = f.n_tokens = f.max_blk = args->n;
    f.n_seqs = pages->n_seqs;
    f.n_groups = n_groups;
    f.max_len = pages->max_pages * pages->page;
    f.heads = F.few_heads = K.heads * F.nsub;
    f.max_cta = min(2 * (uint32_t)ctx->num_sms, kMaxCtas);
    f.min_tiles = kFewMinTiles;
    f.piece_cost = K.e4m3 ? kFewPieceCost8 : kFewPieceCost;
    f.extra = K.e4m3 ? kFewExtra8 : kExtra;
    plan_in g = f;
    g.cu_q = d_group_off;
    g.heads = K.heads;
    g.tok_blk = 2 * R.tq;
    g.max_blk = args->n / g.tok_blk + (n_groups < args->n ? n_groups : args->n);
    g.max_cta = min((uint32_t)ctx->num_sms, kMaxCtas);
    g.min_tiles = kRowsMinTiles;
    g.piece_cost = kRowsPieceCost;
    g.extra = kExtra;

    const bool grouped = n_groups > 0;
    const plan_mem mf(f.max_blk, f.max_cta, f.n, 0, grouped ? (uint64_t)f.n * F.few_heads : 0),
        mg(g.max_blk, g.max_cta, n_groups, grouped ? f.n : 0, grouped ? (uint64_t)f.n * K.heads : 0);
    void *base;
    CR_TRY(cr_scratch(ctx, SCR_ATTN_PLAN, mf.bytes + mg.bytes, &base));
    mf.point(static_cast<char *>(base), f, F);
    mg.point(static_cast<char *>(base) + mf.bytes, g, R);
    CR_TRY(part_mem(ctx, SCR_ATTN_FEW, F, f.max_cta, 16, D));
    if (n_groups) {
        CR_TRY(part_mem(ctx, SCR_ATTN_PART, R, g.max_cta, 2 * kRowsTile, D));
        const size_t heads = (size_t)args->n * args->q_heads, own = (size_t)args->n * F.few_heads * 16;
        void *p;
        CR_TRY(cr_scratch(ctx, SCR_ATTN_PFX, ((heads + own) * (D + 1) + own) * 4, &p));
        F.pfx = R.pfx = static_cast<float *>(p);
        F.own = F.pfx + heads * D;
        F.own_ml = F.own + own * D;
        F.pfx_lse = R.pfx_lse = F.own_ml + 2 * own;
        R.to_pfx = 1;
        F.after_rows = 1;
        CR_TRY(launch_plan<PLAN_FEW>(ctx, f, &g));
        CR_TRY(rows(ctx, R, K, args, g.max_cta));
    } else if (f.n <= kOwnList) {
        F.own_list = 1;
        F.plan = f;
    } else {
        CR_TRY(launch_plan<PLAN_FEW>(ctx, f, nullptr));
    }
    return few(ctx, F, n_groups ? &R : nullptr, K, args, f.max_cta);
}
