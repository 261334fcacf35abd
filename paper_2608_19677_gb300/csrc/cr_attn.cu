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
// pieces in order (k_attn_plan writes the list and the stretches, one CTA).
//
// Two kernels do the work:
//   k_attn_rows  many query rows per key head: 256 rows (tokens x grouped heads) against tiles of
//                128 keys on the tensor cores with accumulators in tensor memory;
//   k_attn_few   at most 16 rows per key head (one token's grouped heads): tiles of 64 keys.
#include <math.h>

#include "cr_internal.cuh"
#include "cr_tensor.cuh"

namespace {

constexpr int kRowsTile = 128;  // query rows of a tile, and keys of one
constexpr int kFewTile = 64;    // keys of a tile of k_attn_few
constexpr int kFewWarps = 4;

// A block of query rows of one key head.
struct __align__(16) attn_blk {
    int row0;   // its first query token
    int ntok;   // its query tokens
    int klen;   // keys of its sequence
    int kbase;  // packed: first key token; paged: row of the table
    int diag;   // keys before the one that its first query token sees last (causal)
    int lo;     // k_attn_few: keys below are already counted (the shared prefix)
    int pad0, pad1;
};
// Where a CTA's stretch begins.
struct __align__(16) attn_start {
    unsigned long long pos;
    uint32_t head, blk, tile, pad[3];
};
struct __align__(16) attn_plan {
    unsigned long long N, Nb;  // key tiles in all, and of one head
    uint32_t nblk, ncta;
    uint32_t pad[2];
};

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
    attn_plan *plan;
    attn_blk *blk;
    unsigned long long *cum;  // [max_blk + 1] key tiles before each block
    attn_start *start;        // [max_cta + 1]
    uint32_t *first;          // [n + 1] first block of each entry
};

enum { PLAN_PACKED, PLAN_PAGED, PLAN_GROUPS, PLAN_FEW };

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// Exclusive scan over the 1,024 threads of the CTA; *total receives the sum.
__device__ unsigned long long scan1024(unsigned long long v, unsigned long long *total)
{
    __shared__ unsigned long long part[32];
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    unsigned long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(~0u, x, o);
        if (lane >= (uint32_t)o) x += y;
    }
    if (lane == 31) part[w] = x;
    __syncthreads();
    if (w == 0) {
        unsigned long long p = part[lane], q = p;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long y = __shfl_up_sync(~0u, q, o);
            if (lane >= (uint32_t)o) q += y;
        }
        part[lane] = q;
    }
    __syncthreads();
    const unsigned long long before = w ? part[w - 1] : 0;
    *total = part[31];
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

// A group's shared keys are read once for all where it has several members.
__device__ __forceinline__ int group_keys(const plan_in &A, uint32_t g)
{
    return A.goff[g + 1] - A.goff[g] >= 2 ? clampi(A.shared[g], 0, (int)A.max_len) : 0;
}

__device__ __forceinline__ uint32_t upper(const unsigned long long *a, uint32_t n, unsigned long long v)
{
    uint32_t lo = 0, hi = n;  // first index with a[] > v
    while (lo < hi) {
        const uint32_t m = (lo + hi) >> 1;
        if (a[m] <= v)
            lo = m + 1;
        else
            hi = m;
    }
    return lo;
}

template <int KIND>
__device__ void plan_build(const plan_in &A, uint32_t *status)
{
    const uint32_t tid = threadIdx.x;
    const uint32_t n = KIND == PLAN_GROUPS ? A.n_groups : A.n;
    unsigned long long total, base = 0;
    // blocks of every entry
    uint32_t nblk;
    if (KIND == PLAN_FEW) {
        nblk = n;
    } else {
        for (uint32_t i0 = 0; i0 < n; i0 += 1024) {
            const uint32_t i = i0 + tid;
            unsigned long long nb = 0;
            if (i < n) {
                int lo, hi;
                q_range(A, i, lo, hi);
                nb = ((uint32_t)(hi - lo) + A.tok_blk - 1) / A.tok_blk;
            }
            const unsigned long long at = base + scan1024(nb, &total);
            if (i < n) A.first[i] = (uint32_t)(at < A.max_blk ? at : A.max_blk);
            base += total;
        }
        if (base > A.max_blk) {  // entries that overlap: not ascending
            if (tid == 0) atomicOr(status, CR_FLAG_BADPAGES);
            base = A.max_blk;
        }
        nblk = (uint32_t)base;
        if (tid == 0) A.first[n] = nblk;
        __syncthreads();
    }
    // their keys
    base = 0;
    for (uint32_t b0 = 0; b0 < nblk; b0 += 1024) {
        const uint32_t b = b0 + tid;
        unsigned long long nt = 0;
        if (b < nblk) {
            uint32_t i = b;
            if (KIND != PLAN_FEW) {
                uint32_t l = 0, h = n;
                while (l < h) {
                    const uint32_t m = (l + h) >> 1;
                    if (A.first[m] <= b)
                        l = m + 1;
                    else
                        h = m;
                }
                i = l - 1;
            }
            attn_blk k = {};
            int lo, hi;
            q_range(A, i, lo, hi);
            if (KIND == PLAN_FEW) {
                k.row0 = (int)i;
                k.ntok = 1;
            } else {
                const int t0 = (int)((b - A.first[i]) * A.tok_blk);
                k.row0 = lo + t0;
                k.ntok = clampi(hi - lo - t0, 0, (int)A.tok_blk);
            }
            if (KIND == PLAN_PACKED) {
                const int klo = clampi(A.cu_k[i], 0, (int)A.n_kv), khi = clampi(A.cu_k[i + 1], klo, (int)A.n_kv);
                k.kbase = klo;
                k.klen = khi - klo;
            } else {
                const uint32_t e = KIND == PLAN_GROUPS ? (uint32_t)lo : i;  // entry whose row is read
                int row = -1;
                if (e < A.n) row = A.seqs ? A.seqs[e] : (int)e;
                if (row < 0 || (uint32_t)row >= A.n_seqs) {
                    if (e < A.n) atomicOr(status, CR_FLAG_BADPAGES);
                    row = -1;
                }
                k.kbase = row < 0 ? 0 : row;
                k.klen = row < 0 ? 0 : clampi(A.lens[row], 0, (int)A.max_len);
                if (KIND == PLAN_GROUPS) {
                    const int s = group_keys(A, i);
                    k.klen = s < k.klen ? s : k.klen;
                }
                if (KIND == PLAN_FEW && A.n_groups) {
                    uint32_t l = 0, h = A.n_groups;  // last group that begins at or before i
                    while (l < h) {
                        const uint32_t m = (l + h) >> 1;
                        if (A.goff[m] <= (int)i)
                            l = m + 1;
                        else
                            h = m;
                    }
                    if (l > 0 && (int)i < A.goff[l]) {
                        // the first member's length bounds what the group's pass has read
                        const uint32_t e0 = (uint32_t)clampi(A.goff[l - 1], 0, (int)A.n - 1);
                        int row0 = A.seqs ? A.seqs[e0] : (int)e0;
                        int s = group_keys(A, l - 1);
                        const int k0 = row0 < 0 || (uint32_t)row0 >= A.n_seqs ? 0 : clampi(A.lens[row0], 0, (int)A.max_len);
                        s = s < k0 ? s : k0;
                        k.lo = s;
                        if (s > k.klen) atomicOr(status, CR_FLAG_BADPAGES);
                    }
                }
            }
            int end = k.klen;
            if (KIND == PLAN_PACKED || KIND == PLAN_PAGED) {
                k.diag = k.klen - (hi - lo) + (k.row0 - lo);
                if (A.causal) end = clampi(k.diag + k.ntok, 0, k.klen);
            }
            if (KIND == PLAN_FEW) {
                const int t = (end + kFewTile - 1) / kFewTile - k.lo / kFewTile;
                nt = t > 1 ? t : 1;
            } else {
                nt = (uint32_t)((end + kRowsTile - 1) / kRowsTile);
                if (nt == 0 && KIND != PLAN_GROUPS) nt = 1;  // rows without keys: zeros
            }
            A.blk[b] = k;
        }
        const unsigned long long at = base + scan1024(nt, &total);
        if (b < nblk) A.cum[b] = at;
        base += total;
    }
    if (tid == 0) A.cum[nblk] = base;
    __syncthreads();
    // stretches
    const unsigned long long Nb = base, N = Nb * A.heads;
    unsigned long long want = N / A.min_tiles;
    const uint32_t ncta = want < 1 ? 1u : (want < A.max_cta ? (uint32_t)want : A.max_cta);
    const unsigned long long snap = N / ncta / 8;  // a stretch ends with its block where that is near
    for (uint32_t c = tid; c <= A.max_cta; c += 1024) {
        attn_start s = {};
        s.pos = c < ncta ? (unsigned long long)((unsigned __int128)N * c / ncta) : N;
        if (s.pos < N) {
            s.head = (uint32_t)(s.pos / Nb);
            const unsigned long long rem = s.pos - s.head * Nb;
            s.blk = upper(A.cum, nblk + 1, rem) - 1;
            const unsigned long long t = rem - A.cum[s.blk], left = A.cum[s.blk + 1] - rem;
            s.tile = (uint32_t)t;
            if (t <= snap) {
                s.pos -= t;
                s.tile = 0;
            } else if (left <= snap) {
                s.pos += left;
                s.tile = 0;
                if (++s.blk == nblk) {
                    s.blk = 0;
                    ++s.head;
                }
            }
        }
        A.start[c] = s;
    }
    if (tid == 0) {
        attn_plan p = {};
        p.N = N;
        p.Nb = Nb;
        p.nblk = nblk;
        p.ncta = ncta;
        *A.plan = p;
    }
}

template <int KIND>
__global__ void __launch_bounds__(1024) k_attn_plan(const __grid_constant__ plan_in a, const __grid_constant__ plan_in b,
                                                    uint32_t *status)
{
    if (blockIdx.x == 0)
        plan_build<KIND>(a, status);
    else
        plan_build<PLAN_GROUPS>(b, status);
}

// What the attention kernels read.
struct attn_in {
    const attn_plan *plan;
    const attn_blk *blk;
    const unsigned long long *cum;
    const attn_start *start;
    const int32_t *table;  // paged
    uint32_t max_pages, page_log2, box_rows, box_log2;
    uint32_t paged, causal, G, nsub, tq, q_heads, head_dim;
    float c;               // scale * log2(e)
    const void *q;         // k_attn_few
    uint64_t q_token, q_head;
    void *o;
    float *lse;
    uint64_t o_token, o_head;
    float *part, *part_ml; // pieces
    float *pfx, *pfx_lse;  // shared prefix: o and log2 of the sum, [token][head]
    uint32_t to_pfx;       // k_attn_rows, its join: write those instead of o
    uint32_t *status;
};

// A CTA's stretch, a block at a time.
struct walk {
    unsigned long long pos, end;
    uint32_t h, b, t0, t1, nt, nblk;
    attn_blk k;
    const attn_in *A;
    __device__ void begin(const attn_in &a)
    {
        A = &a;
        const attn_start s = a.start[blockIdx.x];
        pos = s.pos;
        h = s.head;
        b = s.blk;
        t1 = s.tile;
        end = a.start[blockIdx.x + 1].pos;
        nblk = a.plan->nblk;
    }
    __device__ bool next()
    {
        if (pos >= end) return false;
        for (;;) {
            if (b == nblk) {
                b = 0;
                ++h;
            }
            nt = (uint32_t)(A->cum[b + 1] - A->cum[b]);
            if (nt) break;
            ++b;
        }
        const int4 *g = reinterpret_cast<const int4 *>(A->blk + b);
        int4 *d = reinterpret_cast<int4 *>(&k);
        d[0] = g[0];
        d[1] = g[1];
        t0 = t1;
        const unsigned long long left = end - pos;
        t1 = nt - t0 < left ? nt : t0 + (uint32_t)left;
        pos += t1 - t0;
        return true;
    }
    __device__ void done()
    {
        if (t1 == nt) {
            ++b;
            t1 = 0;
        }
    }
    // scratch place of this piece, or -1: the block is all here
    __device__ int slot() const { return t0 ? 2 * (int)blockIdx.x : (t1 < nt ? 2 * (int)blockIdx.x + 1 : -1); }
};

// ---- many rows --------------------------------------------------------------------------------
// 256 query rows in two tiles of 128 (row r of a tile: token r / G, head r % G of the key head's
// group), one warpgroup of softmax threads each (a thread owns a row), a warp that issues the
// products and one that issues the copies.  Scores of tile X are in columns X*128 .. of tensor
// memory; their weights, 16 bits wide, take the first half of the same columns and are the left
// operand of the product with v, which adds to columns 256 + X*D ...  While one tile's scores are
// in the softmax, the tensor cores work on the other's.
template <int D>
struct rows_cfg {
    static constexpr int kChunks = D / 64;               // 64 elements: a 128-byte row
    static constexpr int kTile = kRowsTile * D * 2;      // bytes of 128 rows
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kStages) * kTile + 1024;
};
// Warps 0-3 and 4-7: softmax; 8: products; 9: copies; 10, 11 only make the warpgroup whole, so that
// its registers can go to the softmax threads (128 scores each): 2 x 128 x 208 + 128 x 80 of the
// launch's 384 x 168.
constexpr int kRowsThreads = 384;

enum { B_QFULL, B_QEMPTY, B_SFULL, B_PREADY = B_SFULL + 2, B_OFULL = B_PREADY + 2, B_OEMPTY = B_OFULL + 2,
       B_DONE = B_OEMPTY + 2, B_FULL };

template <int D, bool BF16>
__global__ void __launch_bounds__(kRowsThreads, 1)
    k_attn_rows(const __grid_constant__ attn_in A, const __grid_constant__ CUtensorMap map_q,
                const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using cfg = rows_cfg<D>;
    extern __shared__ unsigned char dyn[];
    __shared__ __align__(8) unsigned long long bars[B_FULL + 2 * cfg::kStages];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem = (cr_smem(dyn) + 1023u) & ~1023u;
    const uint32_t sq = smem, ring = smem + 2 * cfg::kTile;
    const uint32_t bar = cr_smem(bars);
#define BAR(i) (bar + 8u * (uint32_t)(i))
#define FULL(s) BAR(B_FULL + (s))
#define EMPTY(s) BAR(B_FULL + cfg::kStages + (s))

    if (A.start[blockIdx.x].pos >= A.start[blockIdx.x + 1].pos) return;  // nothing for this CTA
    if (threadIdx.x == 0) {
        gave_up = 0;
        cr_bar_init(BAR(B_QFULL), 1);
        cr_bar_init(BAR(B_QEMPTY), 1);
        cr_bar_init(BAR(B_DONE), 1);
        for (int x = 0; x < 2; ++x) {
            cr_bar_init(BAR(B_SFULL + x), 1);
            cr_bar_init(BAR(B_PREADY + x), 4);
            cr_bar_init(BAR(B_OFULL + x), 1);
            cr_bar_init(BAR(B_OEMPTY + x), 4);
        }
        for (int s = 0; s < cfg::kStages; ++s) {
            cr_bar_init(FULL(s), 1);
            cr_bar_init(EMPTY(s), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // query rows that no copy writes (128 is not a multiple of G) are zeros
    for (uint32_t i = threadIdx.x; i < 2u * cfg::kTile / 16; i += kRowsThreads)
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sq + 16 * i), "r"(0));
    cr_fence_async_smem();
    if (warp == 8) cr_tmem_alloc(cr_smem(&tmem_at), 512);
    cr_tc_before();
    __syncthreads();
    cr_tc_after();
    const uint32_t tmem = tmem_at;

    walk w;
    w.begin(A);
    const uint32_t q_bytes = A.G * A.tq * 128 * cfg::kChunks;

    if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 9) {
        // ---- copies ----
        if (lane == 0) {
            cr_tma_prefetch_map(&map_q);
            cr_tma_prefetch_map(&map_k);
            cr_tma_prefetch_map(&map_v);
        }
        uint32_t stage = 0, phase = 0, qphase = 0;
        while (w.next()) {
            const int two = w.k.ntok > (int)A.tq;
            if (!cr_bar_wait(BAR(B_QEMPTY), qphase ^ 1, &gave_up)) goto out;
            qphase ^= 1;
            if (lane == 0) {
                cr_bar_expect(BAR(B_QFULL), q_bytes * (1 + two));
                for (int x = 0; x <= two; ++x)
                    for (int ch = 0; ch < cfg::kChunks; ++ch)
                        cr_tma_load(sq + x * cfg::kTile + ch * (kRowsTile * 128), &map_q, BAR(B_QFULL), ch * 64, 0,
                                    (int)w.h, w.k.row0 + x * (int)A.tq);
            }
            // lane: one box of one column block of a tile
            const uint32_t boxes = kRowsTile >> A.box_log2;
            const uint32_t box = lane & (boxes - 1), ch = lane / boxes;
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                const int key = (int)(t * kRowsTile + (box << A.box_log2));
                // packed keys come as one box; its rows behind the sequence are never used
                const bool on = lane < boxes * cfg::kChunks && (!A.paged || key < w.k.klen);
                const uint32_t bytes = __popc(__ballot_sync(~0u, on)) * A.box_rows * 128;
                int y, pg = 0;
                if (A.paged) {
                    const uint32_t pi = (uint32_t)key >> A.page_log2;
                    if (on) pg = __ldg(A.table + (uint64_t)w.k.kbase * A.max_pages + pi);
                    y = key & ((1 << A.page_log2) - 1);
                } else {
                    y = w.k.kbase + key;
                }
                for (int v = 0; v < 2; ++v) {
                    if (!cr_bar_wait(EMPTY(stage), phase ^ 1, &gave_up)) goto out;
                    if (lane == 0) cr_bar_expect(FULL(stage), bytes);
                    __syncwarp();
                    if (on)
                        cr_tma_load(ring + stage * cfg::kTile + ch * (kRowsTile * 128) + ((box << A.box_log2) * 128),
                                    v ? &map_v : &map_k, FULL(stage), (int)ch * 64, y, (int)w.h, pg);
                    if (++stage == cfg::kStages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
            }
            w.done();
        }
    } else if (warp == 8) {
        // ---- products ----
        if (lane == 0) {
            const uint32_t id_s = cr_idesc(BF16, 128, 128, false), id_o = cr_idesc(BF16, 128, D, true);
            uint32_t stage = 0, phase = 0, qphase = 0, pphase[2] = {0, 0}, ophase[2] = {0, 0};
            auto scores = [&](int x, uint32_t st) {
                const uint32_t a = sq + x * cfg::kTile, b = ring + st * cfg::kTile;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t off = (i / 4) * (kRowsTile * 128) + (i % 4) * 32;
                    cr_mma_ss(tmem + x * 128, cr_sdesc(a + off, 16, 1024), cr_sdesc(b + off, 16, 1024), id_s, i > 0);
                }
            };
            auto values = [&](int x, uint32_t st, bool first) {
                const uint32_t b = ring + st * cfg::kTile;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    cr_mma_ts(tmem + 256 + x * D, tmem + x * 128 + i * 8,
                              cr_sdesc(b + i * 2048, kRowsTile * 128, 1024), id_o, !(first && i == 0));
            };
            while (w.next()) {
                const int two = w.k.ntok > (int)A.tq;
                const uint32_t n = w.t1 - w.t0;
                if (!cr_bar_wait(BAR(B_QFULL), qphase, &gave_up)) goto out;
                qphase ^= 1;
                if (!cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
                cr_tc_after();
                for (int x = 0; x <= two; ++x) {
                    scores(x, stage);
                    cr_tc_commit(BAR(B_SFULL + x));
                }
                cr_tc_commit(EMPTY(stage));
                if (n == 1) cr_tc_commit(BAR(B_QEMPTY));
                if (++stage == cfg::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
                for (uint32_t j = 0; j < n; ++j) {
                    const uint32_t vs = stage;
                    if (!cr_bar_wait(FULL(vs), phase, &gave_up)) goto out;
                    if (++stage == cfg::kStages) {
                        stage = 0;
                        phase ^= 1;
                    }
                    const uint32_t ks = stage;
                    const bool more = j + 1 < n;
                    if (more) {
                        if (!cr_bar_wait(FULL(ks), phase, &gave_up)) goto out;
                        if (++stage == cfg::kStages) {
                            stage = 0;
                            phase ^= 1;
                        }
                    }
                    for (int x = 0; x <= two; ++x) {
                        if (j == 0) {
                            if (!cr_bar_wait(BAR(B_OEMPTY + x), ophase[x] ^ 1, &gave_up)) goto out;
                            ophase[x] ^= 1;
                        }
                        if (!cr_bar_wait(BAR(B_PREADY + x), pphase[x], &gave_up)) goto out;
                        pphase[x] ^= 1;
                        cr_tc_after();
                        values(x, vs, j == 0);
                        if (more) {
                            scores(x, ks);
                            cr_tc_commit(BAR(B_SFULL + x));
                        } else {
                            cr_tc_commit(BAR(B_OFULL + x));
                        }
                    }
                    cr_tc_commit(EMPTY(vs));
                    if (more) {
                        cr_tc_commit(EMPTY(ks));
                        if (j + 2 == n) cr_tc_commit(BAR(B_QEMPTY));
                    }
                }
                w.done();
            }
            cr_tc_commit(BAR(B_DONE));  // the shared memory is in use until the last product has ended
            cr_bar_wait(BAR(B_DONE), 0, &gave_up);
        }
    } else if (warp < 8) {
        // ---- softmax: a thread owns a row ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int x = (int)(warp >> 2);
        const uint32_t row = threadIdx.x & 127;
        const uint32_t lanes = (warp & 3) << 21;  // this warp's lanes of tensor memory
        const uint32_t ts = tmem + x * 128 + lanes, to = tmem + 256 + x * D + lanes;
        const int tok = (int)(row / A.G), g = (int)(row % A.G);
        const float c = A.c;
        const unsigned long long c2 = cr_pair(c, c);
        uint32_t sphase = 0, ophase = 0, stage = 0, phase = 0;  // stage, phase: of the piece's first key tile
        while (w.next()) {
            const int two = w.k.ntok > (int)A.tq;
            const uint32_t n = w.t1 - w.t0;
            if (x <= two) {
                const int mine = x * (int)A.tq + tok;  // token of the block
                const bool valid = row < A.G * A.tq && mine < w.k.ntok;
                int lim = w.k.klen;  // keys that this row sees
                if (A.causal) lim = min(lim, w.k.diag + mine + 1);
                float m = -INFINITY, l = 0.f;
                for (uint32_t j = 0; j < n; ++j) {
                    const int k0 = (int)(w.t0 + j) * kRowsTile;
                    if (!cr_bar_wait(BAR(B_SFULL + x), sphase, &gave_up)) goto out;
                    sphase ^= 1;
                    cr_tc_after();
                    uint32_t s[128];
#pragma unroll
                    for (int i = 0; i < 4; ++i) cr_tmem_ld(ts + 32 * i, s + 32 * i);
                    cr_tmem_ld_wait();
                    const int seen = lim - k0;
                    if (__any_sync(~0u, seen < kRowsTile)) {
#pragma unroll
                        for (int i = 0; i < 128; ++i) s[i] = i < seen ? s[i] : 0xff800000u;
                    }
                    float mx[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        mx[i] = __uint_as_float(s[i]);
#pragma unroll
                        for (int e = 4; e < 124; e += 8)
                            mx[i] = cr_max3(mx[i], __uint_as_float(s[e + i]), __uint_as_float(s[e + 4 + i]));
                        mx[i] = fmaxf(mx[i], __uint_as_float(s[124 + i]));
                    }
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    // The maximum may lag by 2^8: weights stay below 2^8, sums below 2^31, and the
                    // accumulator is scaled a few times per row instead of at every tile.
                    const bool grow = j == 0 || !((top - m) * c <= 8.f || top == m);
                    if (__any_sync(~0u, grow)) {
                        const float m_new = fmaxf(m, top);
                        if (j > 0) {
                            const float f = m_new == m ? 1.f : cr_exp2((m - m_new) * c);
                            l *= f;
#pragma unroll 1
                            for (int i = 0; i < D / 32; ++i) {
                                uint32_t o[32];
                                cr_tmem_ld(to + 32 * i, o);
                                cr_tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                cr_tmem_st(to + 32 * i, o);
                            }
                            cr_tmem_st_wait();
                        }
                        m = m_new;
                    }
                    const float off = m == -INFINITY ? 0.f : -m * c;
                    const unsigned long long off2 = cr_pair(off, off);
                    unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < 128; i += 64) {
                        uint32_t p[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            float a, b;
                            cr_unpair(cr_fma2(cr_pair(__uint_as_float(s[i + 2 * e]), __uint_as_float(s[i + 2 * e + 1])), c2,
                                              off2),
                                      a, b);
                            a = cr_exp2(a);
                            b = cr_exp2(b);
                            sum[e & 1] = cr_add2(sum[e & 1], cr_pair(a, b));
                            p[e] = cr_pack16<BF16>(a, b);
                        }
                        cr_tmem_st(ts + i / 2, p);
                    }
                    float s0, s1;
                    cr_unpair(cr_add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    // keys behind the sequence's end have weight zero, but what stands there may be
                    // no number: their rows of v become zeros
                    if (x == 0 && k0 + kRowsTile > w.k.klen) {
                        const uint32_t at = stage + 2 * j + 1;
                        const uint32_t st = at % cfg::kStages, ph = phase ^ ((at / cfg::kStages) & 1);
                        if (!cr_bar_wait(FULL(st), ph, &gave_up)) goto out;
                        if (k0 + (int)row >= w.k.klen) {
#pragma unroll
                            for (int i = 0; i < D / 8; ++i)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(
                                                 ring + st * cfg::kTile + (i / 8) * (kRowsTile * 128) + row * 128 + (i % 8) * 16),
                                             "r"(0)
                                             : "memory");
                        }
                        cr_fence_async_smem();
                    }
                    cr_tmem_st_wait();
                    cr_tc_before();
                    __syncwarp();
                    if (lane == 0) cr_bar_arrive(BAR(B_PREADY + x));
                }
                // ---- the piece's result ----
                if (!cr_bar_wait(BAR(B_OFULL + x), ophase, &gave_up)) goto out;
                ophase ^= 1;
                cr_tc_after();
                const int slot = w.slot();
                const int head = (int)(w.h * A.G) + g;
                const uint64_t tk = (uint64_t)(w.k.row0 + mine);
                if (slot >= 0) {
                    const uint64_t at = (uint64_t)(2 * slot + x);
                    float4 *dst = reinterpret_cast<float4 *>(A.part) + at * (D / 4) * kRowsTile + row;
#pragma unroll 1
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t o[32];
                        cr_tmem_ld(to + 32 * i, o);
                        cr_tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            dst[(i * 8 + e) * kRowsTile] =
                                make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]),
                                            __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    }
                    reinterpret_cast<float2 *>(A.part_ml)[at * kRowsTile + row] =
                        make_float2(m == -INFINITY ? m : m * c, l);
                } else {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    const float lse2 = l == 0.f ? -INFINITY : m * c + log2f(l);
#pragma unroll 1
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t o[32];
                        cr_tmem_ld(to + 32 * i, o);
                        cr_tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            o[e] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv);
                        if (!valid) continue;
                        if (A.to_pfx) {
                            float *dst = A.pfx + (tk * A.q_heads + head) * D + 32 * i;
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                *reinterpret_cast<uint4 *>(dst + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                        } else {
                            uint16_t *dst = static_cast<uint16_t *>(A.o) + tk * A.o_token + head * A.o_head + 32 * i;
#pragma unroll
                            for (int e = 0; e < 32; e += 8)
                                if (32 * i + e < (int)A.head_dim) {
                                    uint4 v;
                                    v.x = cr_pack16<BF16>(__uint_as_float(o[e]), __uint_as_float(o[e + 1]));
                                    v.y = cr_pack16<BF16>(__uint_as_float(o[e + 2]), __uint_as_float(o[e + 3]));
                                    v.z = cr_pack16<BF16>(__uint_as_float(o[e + 4]), __uint_as_float(o[e + 5]));
                                    v.w = cr_pack16<BF16>(__uint_as_float(o[e + 6]), __uint_as_float(o[e + 7]));
                                    *reinterpret_cast<uint4 *>(dst + e) = v;
                                }
                        }
                    }
                    if (valid) {
                        if (A.to_pfx)
                            A.pfx_lse[tk * A.q_heads + head] = lse2;
                        else if (A.lse)
                            A.lse[tk * A.q_heads + head] = lse2 * 0.693147180559945309f;
                    }
                }
                cr_tc_before();
                __syncwarp();
                if (lane == 0) cr_bar_arrive(BAR(B_OEMPTY + x));
            }
            stage += 2 * n;
            phase ^= (stage / cfg::kStages) & 1;
            stage %= cfg::kStages;
            w.done();
        }
    }
out:
    __syncwarp();
    if (gave_up) {  // let the copies and products that are under way end
        if (threadIdx.x == 0) atomicOr(A.status, CR_FLAG_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    cr_tc_before();
    __syncthreads();
    if (warp == 8) {
        cr_tc_after();
        cr_tmem_free(tmem, 512);
    }
#undef FULL
#undef EMPTY
#undef BAR
}

// First stretch that begins inside a block: true for the CTA that joins the block's pieces.
__device__ __forceinline__ bool join_here(const attn_in &A, uint32_t c, attn_start &s, unsigned long long &begin,
                                          unsigned long long &end)
{
    if (c == 0 || c >= A.plan->ncta) return false;
    s = A.start[c];
    if (s.pos >= A.plan->N || s.tile == 0) return false;
    begin = s.pos - s.tile;
    end = begin + (A.cum[s.blk + 1] - A.cum[s.blk]);
    return A.start[c - 1].pos <= begin;
}

// Joins the pieces of blocks that several CTAs worked on: blockIdx.x + 1 is the stretch that begins
// inside the block, blockIdx.y 32 of its rows.  A thread joins four columns of one row at a time.
template <int D, bool BF16>
__global__ void __launch_bounds__(256) k_attn_rows_join(const __grid_constant__ attn_in A)
{
    const uint32_t c = blockIdx.x + 1;
    attn_start s;
    unsigned long long begin, end;
    if (!join_here(A, c, s, begin, end)) return;
    const attn_blk k = A.blk[s.blk];
    const uint32_t x = blockIdx.y >> 2, row = (blockIdx.y & 3) * 32 + (threadIdx.x & 31);
    const int tok = (int)(x * A.tq + row / A.G);
    if (row >= A.G * A.tq || tok >= k.ntok) return;
    const float2 *ml = reinterpret_cast<const float2 *>(A.part_ml);
    const float4 *part = reinterpret_cast<const float4 *>(A.part);
    float m = -INFINITY;
    for (uint32_t p = c - 1; A.start[p].pos < end; ++p) {
        if (A.start[p].pos == A.start[p + 1].pos) continue;
        const uint64_t at = 2ull * (p == c - 1 ? 2 * p + 1 : 2 * p) + x;
        m = fmaxf(m, ml[at * kRowsTile + row].x);
    }
    const int head = (int)(s.head * A.G + row % A.G);
    const uint64_t tk = (uint64_t)(k.row0 + tok);
    for (uint32_t d4 = threadIdx.x >> 5; d4 < D / 4; d4 += 8) {
        float l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t p = c - 1; A.start[p].pos < end; ++p) {
            if (A.start[p].pos == A.start[p + 1].pos) continue;
            const uint64_t at = 2ull * (p == c - 1 ? 2 * p + 1 : 2 * p) + x;
            const float2 q = ml[at * kRowsTile + row];
            if (q.x == -INFINITY) continue;  // sees none of these keys
            const float f = cr_exp2(q.x - m);
            const float4 v = part[(at * (D / 4) + d4) * kRowsTile + row];
            l += q.y * f;
            o.x += v.x * f;
            o.y += v.y * f;
            o.z += v.z * f;
            o.w += v.w * f;
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
        if (A.to_pfx) {
            *reinterpret_cast<float4 *>(A.pfx + (tk * A.q_heads + head) * D + 4 * d4) = o;
            if (d4 == 0) A.pfx_lse[tk * A.q_heads + head] = lse2;
        } else {
            if (4 * d4 < A.head_dim)
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.o) + tk * A.o_token + head * A.o_head + 4 * d4) =
                    make_uint2(cr_pack16<BF16>(o.x, o.y), cr_pack16<BF16>(o.z, o.w));
            if (d4 == 0 && A.lse) A.lse[tk * A.q_heads + head] = lse2 * 0.693147180559945309f;
        }
    }
}

// ---- few rows ---------------------------------------------------------------------------------
// One token's query heads of a key head, 16 at most.  Here the bytes of k and v are the bound
// (each is used for a few rows only), so the small register-operand products do: four warps take
// 16 keys each of a tile of 64 that a fifth warp's copies bring, with the softmax state of the
// rows in every warp, joined at the piece's end.
template <int D, bool WIDE>
struct few_cfg {
    static constexpr int kChunks = D / 64;
    static constexpr int kTile = kFewTile * D * 2;  // bytes of 64 keys
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kJoin = kFewWarps * 8 * D * 4;  // eight rows of every warp
    static constexpr int kSmem = kStages * 2 * kTile + kJoin + 1024;
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
    k_attn_few(const __grid_constant__ attn_in A, const __grid_constant__ CUtensorMap map_k,
               const __grid_constant__ CUtensorMap map_v)
{
    using cfg = few_cfg<D, WIDE>;
    extern __shared__ unsigned char dyn[];
    __shared__ __align__(8) unsigned long long bars[2 * cfg::kStages];
    __shared__ float2 join_ml[kFewWarps][16];
    __shared__ int gave_up;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = cr_smem(dyn), ring = (base + 1023u) & ~1023u;
    float *join = reinterpret_cast<float *>(dyn + (ring - base) + cfg::kStages * 2 * cfg::kTile);
    const uint32_t bar = cr_smem(bars);
#define FULL(s) (bar + 8u * (s))
#define EMPTY(s) (bar + 8u * (cfg::kStages + (s)))

    if (A.start[blockIdx.x].pos >= A.start[blockIdx.x + 1].pos) return;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int s = 0; s < cfg::kStages; ++s) {
            cr_bar_init(FULL(s), 1);
            cr_bar_init(EMPTY(s), kFewWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();

    walk w;
    w.begin(A);
    uint32_t stage = 0, phase = 0;
    if (warp == kFewWarps) {
        // ---- copies: a lane brings one box of one column block, keys then values ----
        const uint32_t boxes = kFewTile >> A.box_log2;
        const uint32_t box = lane & (boxes - 1), ch = lane / boxes;
        while (w.next()) {
            const int kv = (int)(w.h / A.nsub);
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                const int key = (int)((w.k.lo / kFewTile + t) * kFewTile + (box << A.box_log2));
                const bool on = lane < boxes * cfg::kChunks && key < w.k.klen;
                const uint32_t bytes = 2 * __popc(__ballot_sync(~0u, on)) * A.box_rows * 128;
                int pg = 0;
                if (on) pg = __ldg(A.table + (uint64_t)w.k.kbase * A.max_pages + ((uint32_t)key >> A.page_log2));
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
            w.done();
        }
    } else {
        const uint32_t r4 = lane >> 2, q4 = lane & 3;
        const float c = A.c;
        while (w.next()) {
            const uint32_t kv = w.h / A.nsub, sub = w.h % A.nsub;
            const uint32_t h0 = kv * A.G + sub * 16;                       // first query head of the rows
            const uint32_t rows = min(16u, A.G - sub * 16);
            const uint16_t *q = static_cast<const uint16_t *>(A.q) + (uint64_t)w.k.row0 * A.q_token;
            uint32_t qa[D / 16][4];
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t r = r4 + (e & 1) * 8, d = i * 16 + q4 * 2 + (e >> 1) * 8;
                    qa[i][e] = 0;
                    if ((WIDE || !(e & 1)) && r < rows && d < A.head_dim)
                        qa[i][e] = *reinterpret_cast<const uint32_t *>(q + (uint64_t)(h0 + r) * A.q_head + d);
                }
            float o[D / 8][4];
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
            float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
            for (uint32_t t = w.t0; t < w.t1; ++t) {
                if (!cr_bar_wait(FULL(stage), phase, &gave_up)) goto out;
                const int key = (int)((w.k.lo / kFewTile + t) * kFewTile + warp * 16);  // this warp's first key
                if (key < w.k.klen && key + 16 > w.k.lo) {
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
                    if (key + 16 > w.k.klen || key < w.k.lo) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int j = key + i * 8 + (int)q4 * 2 + e;
                                if (j < w.k.lo || j >= w.k.klen) {
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
                        const float off = m[r] == -INFINITY ? 0.f : -m[r] * c;
                        float p[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] = cr_exp2(fmaf(s[i >> 1][2 * r + (i & 1)], c, off));
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
            // ---- the four warps' states join, eight rows at a time ----
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                l[r] += __shfl_xor_sync(~0u, l[r], 1);
                l[r] += __shfl_xor_sync(~0u, l[r], 2);
                if (q4 == 0) join_ml[warp][r4 + 8 * r] = make_float2(m[r] == -INFINITY ? m[r] : m[r] * c, l[r]);
            }
            const int slot = w.slot();
            const bool from_pfx = w.k.lo > 0 && w.t0 == 0;
#pragma unroll
            for (int r = 0; r < (WIDE ? 2 : 1); ++r) {
                if (rows <= 8u * r) break;
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    *reinterpret_cast<float2 *>(join + (warp * 8 + r4) * D + i * 8 + q4 * 2) =
                        make_float2(o[i][2 * r], o[i][2 * r + 1]);
                asm volatile("bar.sync 1, 128;" ::: "memory");
                for (uint32_t e = threadIdx.x; e < 8 * D / 4; e += 128) {
                    const uint32_t rr = e / (D / 4), d4 = e % (D / 4), row = 8 * r + rr;
                    if (row >= rows) continue;
                    const uint64_t oh = (uint64_t)w.k.row0 * A.q_heads + h0 + row;
                    float mm = -INFINITY, ll = 0.f;
                    for (int v = 0; v < kFewWarps; ++v) mm = fmaxf(mm, join_ml[v][row].x);
                    float px = -INFINITY;
                    if (from_pfx) {
                        px = A.pfx_lse[oh];
                        mm = fmaxf(mm, px);
                    }
                    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int v = 0; v < kFewWarps; ++v) {
                        const float2 ml = join_ml[v][row];
                        if (ml.x == -INFINITY) continue;
                        const float f = cr_exp2(ml.x - mm);
                        const float4 x = *reinterpret_cast<const float4 *>(join + (v * 8 + rr) * D + 4 * d4);
                        ll += ml.y * f;
                        s.x += x.x * f;
                        s.y += x.y * f;
                        s.z += x.z * f;
                        s.w += x.w * f;
                    }
                    if (px != -INFINITY) {
                        const float f = cr_exp2(px - mm);
                        const float4 x = *reinterpret_cast<const float4 *>(A.pfx + oh * D + 4 * d4);
                        ll += f;
                        s.x += x.x * f;
                        s.y += x.y * f;
                        s.z += x.z * f;
                        s.w += x.w * f;
                    }
                    if (slot >= 0) {
                        const uint64_t at = (uint64_t)slot * 16 + row;
                        *reinterpret_cast<float4 *>(A.part + at * D + 4 * d4) = s;
                        if (d4 == 0) reinterpret_cast<float2 *>(A.part_ml)[at] = make_float2(mm, ll);
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
                asm volatile("bar.sync 1, 128;" ::: "memory");
            }
            w.done();
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
}

// Joins the pieces of blocks that several CTAs of k_attn_few worked on: 16 rows by D columns.
template <int D, bool BF16>
__global__ void __launch_bounds__(128) k_attn_few_join(const __grid_constant__ attn_in A)
{
    const uint32_t c = blockIdx.x + 1;
    attn_start s;
    unsigned long long begin, end;
    if (!join_here(A, c, s, begin, end)) return;
    const attn_blk k = A.blk[s.blk];
    const uint32_t kv = s.head / A.nsub, sub = s.head % A.nsub;
    const uint32_t h0 = kv * A.G + sub * 16, rows = min(16u, A.G - sub * 16);
    const float2 *ml = reinterpret_cast<const float2 *>(A.part_ml);
    for (uint32_t e = threadIdx.x; e < rows * (D / 4); e += 128) {
        const uint32_t row = e / (D / 4), d4 = e % (D / 4);
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t p = c - 1; A.start[p].pos < end; ++p)
            if (A.start[p].pos != A.start[p + 1].pos)
                m = fmaxf(m, ml[(uint64_t)(p == c - 1 ? 2 * p + 1 : 2 * p) * 16 + row].x);
        for (uint32_t p = c - 1; A.start[p].pos < end; ++p) {
            if (A.start[p].pos == A.start[p + 1].pos) continue;
            const uint64_t at = (uint64_t)(p == c - 1 ? 2 * p + 1 : 2 * p) * 16 + row;
            const float2 q = ml[at];
            if (q.x == -INFINITY) continue;
            const float f = cr_exp2(q.x - m);
            const float4 v = *reinterpret_cast<const float4 *>(A.part + at * D + 4 * d4);
            l += q.y * f;
            o.x += v.x * f;
            o.y += v.y * f;
            o.z += v.z * f;
            o.w += v.w * f;
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (4 * d4 < A.head_dim)
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.o) + (uint64_t)k.row0 * A.o_token +
                                       (uint64_t)(h0 + row) * A.o_head + 4 * d4) =
                make_uint2(cr_pack16<BF16>(o.x * inv, o.y * inv), cr_pack16<BF16>(o.z * inv, o.w * inv));
        if (d4 == 0 && A.lse)
            A.lse[(uint64_t)k.row0 * A.q_heads + h0 + row] = (l == 0.f ? -INFINITY : m + log2f(l)) * 0.693147180559945309f;
    }
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
// 64 elements of the first.
int encode_map(cr_ctx *ctx, CUtensorMap *map, bool bf16, const void *base, const uint64_t dim[4], const uint64_t stride[3],
               const uint32_t box[3], bool stream_once)
{
    encode_fn fn = encoder();
    if (!fn) return cr_fail(ctx, CR_ECUDA, "cuTensorMapEncodeTiled is not available from this driver");
    cuuint64_t st[3];
    for (int i = 0; i < 3; ++i) st[i] = dim[i + 1] == 1 ? 16 : stride[i] * 2;  // never stepped over
    const cuuint32_t bx[4] = {64, box[0], box[1], box[2]}, es[4] = {1, 1, 1, 1};
    const cuuint64_t dm[4] = {dim[0], dim[1], dim[2], dim[3]};
    const CUresult r = fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                          const_cast<void *>(base), dm, st, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B,
                          stream_once ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cr_fail(ctx, CR_EINVAL, "tensor map rejected (%d): check pointers and strides", (int)r);
    return CR_OK;
}

// Keys and values of a call.
struct kv_desc {
    bool paged, bf16;
    uint32_t heads, dim;
    const void *k, *v;
    uint64_t k_row, k_head, v_row, v_head;  // elements between tokens, heads
    // packed
    uint32_t n_kv;
    const int32_t *cu_k;
    // paged
    const cr_kv_pages *pg;
};

int kv_map(cr_ctx *ctx, CUtensorMap *map, const kv_desc &K, bool value, uint32_t box_rows)
{
    uint64_t dim[4] = {K.dim, 0, K.heads, 1}, st[3] = {value ? K.v_row : K.k_row, value ? K.v_head : K.k_head, 8};
    if (K.paged) {
        dim[1] = K.pg->page;
        dim[3] = K.pg->n_pages;
        st[2] = K.pg->page_stride;
    } else {
        dim[1] = K.n_kv;
    }
    const uint32_t box[3] = {box_rows, 1, 1};
    return encode_map(ctx, map, K.bf16, value ? K.v : K.k, dim, st, box, K.paged);
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
    size_t plan, blk, cum, start, first;
    plan_mem(uint32_t max_blk, uint32_t max_cta, uint32_t n)
    {
        bytes = 0;
        auto take = [&](size_t b) {
            const size_t at = bytes;
            bytes += (b + 255) & ~(size_t)255;
            return at;
        };
        plan = take(sizeof(attn_plan));
        blk = take(sizeof(attn_blk) * ((size_t)max_blk + 1));
        cum = take(8 * ((size_t)max_blk + 2));
        start = take(sizeof(attn_start) * ((size_t)max_cta + 2));
        first = take(4 * ((size_t)n + 1));
    }
    void point(char *base, plan_in &p, attn_in &a) const
    {
        p.plan = reinterpret_cast<attn_plan *>(base + plan);
        p.blk = reinterpret_cast<attn_blk *>(base + blk);
        p.cum = reinterpret_cast<unsigned long long *>(base + cum);
        p.start = reinterpret_cast<attn_start *>(base + start);
        p.first = reinterpret_cast<uint32_t *>(base + first);
        a.plan = p.plan;
        a.blk = p.blk;
        a.cum = p.cum;
        a.start = p.start;
    }
};

bool aligned(const void *p, uint64_t a, uint64_t b) { return ((uintptr_t)p & 15) == 0 && (a & 7) == 0 && (b & 7) == 0; }

int check_heads(cr_ctx *ctx, const char *who, const cr_attn_args *a, uint32_t dtype, uint32_t kv_heads, uint32_t dim)
{
    if (dtype > CR_DTYPE_FP16) return cr_fail(ctx, CR_EINVAL, "%s: dtype %u", who, dtype);
    if (kv_heads == 0 || kv_heads > 65536 || a->q_heads == 0 || a->q_heads % kv_heads || a->q_heads / kv_heads > 128)
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
    A.head_dim = K.dim;
    A.c = a->scale * 1.44269504088896341f;
    A.causal = a->causal != 0;
    A.q = a->d_q;
    A.q_token = a->q_token;
    A.q_head = a->q_head;
    A.o = a->d_o;
    A.o_token = a->o_token;
    A.o_head = a->o_head;
    A.lse = a->d_lse;
    A.status = ctx->d_status;
    if (K.paged) {
        A.table = K.pg->d_table;
        A.max_pages = K.pg->max_pages;
        A.page_log2 = ilog2(K.pg->page);
    }
}

template <int D, bool BF16>
int launch_rows(cr_ctx *ctx, const attn_in &A, const kv_desc &K, const cr_attn_args *a, uint32_t ctas, bool join)
{
    CUtensorMap mq, mk, mv;
    const uint64_t dim[4] = {K.dim, A.G, K.heads, a->n_tokens}, st[3] = {a->q_head, a->q_head * A.G, a->q_token};
    const uint32_t box[3] = {A.G, 1, A.tq};
    CR_TRY(encode_map(ctx, &mq, BF16, a->d_q, dim, st, box, false));
    CR_TRY(kv_map(ctx, &mk, K, false, A.box_rows));
    CR_TRY(kv_map(ctx, &mv, K, true, A.box_rows));
    auto kern = k_attn_rows<D, BF16>;
    CR_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, rows_cfg<D>::kSmem));
    CR_LAUNCH(ctx, kern, ctas, kRowsThreads, rows_cfg<D>::kSmem, A, mq, mk, mv);
    if (join && ctas > 1) {
        auto kj = k_attn_rows_join<D, BF16>;
        CR_LAUNCH(ctx, kj, dim3(ctas - 1, 8), 256, 0, A);
    }
    return CR_OK;
}

int rows(cr_ctx *ctx, const attn_in &A, const kv_desc &K, const cr_attn_args *a, uint32_t ctas)
{
    if (K.dim <= 64)
        return K.bf16 ? launch_rows<64, true>(ctx, A, K, a, ctas, true) : launch_rows<64, false>(ctx, A, K, a, ctas, true);
    return K.bf16 ? launch_rows<128, true>(ctx, A, K, a, ctas, true) : launch_rows<128, false>(ctx, A, K, a, ctas, true);
}

template <int D, bool BF16, bool WIDE>
int launch_few(cr_ctx *ctx, const attn_in &A, const kv_desc &K, uint32_t ctas)
{
    CUtensorMap mk, mv;
    CR_TRY(kv_map(ctx, &mk, K, false, A.box_rows));
    CR_TRY(kv_map(ctx, &mv, K, true, A.box_rows));
    auto kern = k_attn_few<D, BF16, WIDE>;
    CR_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, few_cfg<D, WIDE>::kSmem));
    CR_LAUNCH(ctx, kern, ctas, kFewThreads, (few_cfg<D, WIDE>::kSmem), A, mk, mv);
    if (ctas > 1) {
        auto kj = k_attn_few_join<D, BF16>;
        CR_LAUNCH(ctx, kj, ctas - 1, 128, 0, A);
    }
    return CR_OK;
}

int few(cr_ctx *ctx, const attn_in &A, const kv_desc &K, uint32_t ctas)
{
    const bool wide = A.G > 8;
    if (K.dim <= 64) {
        if (K.bf16) return wide ? launch_few<64, true, true>(ctx, A, K, ctas) : launch_few<64, true, false>(ctx, A, K, ctas);
        return wide ? launch_few<64, false, true>(ctx, A, K, ctas) : launch_few<64, false, false>(ctx, A, K, ctas);
    }
    if (K.bf16) return wide ? launch_few<128, true, true>(ctx, A, K, ctas) : launch_few<128, true, false>(ctx, A, K, ctas);
    return wide ? launch_few<128, false, true>(ctx, A, K, ctas) : launch_few<128, false, false>(ctx, A, K, ctas);
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

constexpr uint32_t kRowsMinTiles = 4, kFewMinTiles = 4;

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
    if (K.paged) {
        p.lens = K.pg->d_lens;
        p.n_seqs = K.pg->n_seqs;
        p.max_len = K.pg->max_pages * K.pg->page;
    }
    p.max_cta = (uint32_t)ctx->num_sms;
    const plan_mem mem(p.max_blk, p.max_cta, a->n);
    void *base;
    CR_TRY(cr_scratch(ctx, SCR_ATTN_PLAN, mem.bytes, &base));
    mem.point(static_cast<char *>(base), p, A);
    CR_TRY(part_mem(ctx, SCR_ATTN_PART, A, p.max_cta, 2 * kRowsTile, K.dim <= 64 ? 64 : 128));
    if (K.paged)
        CR_LAUNCH(ctx, k_attn_plan<PLAN_PAGED>, 1, 1024, 0, p, p, ctx->d_status);
    else
        CR_LAUNCH(ctx, k_attn_plan<PLAN_PACKED>, 1, 1024, 0, p, p, ctx->d_status);
    return rows(ctx, A, K, a, p.max_cta);
}

}  // namespace

// Limits of a pool of pages (cr_pages.cu).
int cr_pages_check(cr_ctx *ctx, const char *who, const cr_kv_pages *pg);

static int paged_desc(cr_ctx *ctx, const char *who, const cr_kv_pages *pg, uint32_t layer, kv_desc &K)
{
    CR_TRY(cr_pages_check(ctx, who, pg));
    if (layer >= pg->layers) return cr_fail(ctx, CR_EINVAL, "%s: layer %u of %u", who, layer, pg->layers);
    K = kv_desc{};
    K.paged = true;
    K.bf16 = pg->dtype == CR_DTYPE_BF16;
    K.heads = pg->kv_heads;
    K.dim = pg->head_dim;
    K.k = static_cast<const uint16_t *>(pg->d_cache) + layer * pg->layer_stride;
    K.v = static_cast<const uint16_t *>(K.k) + pg->kv_stride;
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
    if (n_kv == 0) {  // nothing to map: any 16-byte aligned memory stands for the empty tensors
        K.k = K.v = args->d_q;
        K.k_row = K.v_row = args->q_token;
        K.k_head = K.v_head = 8;
        K.heads = kv_heads;
    }
    return attn_many(ctx, args, K);
}

extern "C" int cr_attn_paged(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, const cr_attn_args *args)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_attn_paged");
    if (!args) return cr_fail(ctx, CR_EINVAL, "cr_attn_paged: args is NULL");
    kv_desc K;
    CR_TRY(paged_desc(ctx, "cr_attn_paged", pages, layer, K));
    CR_TRY(check_heads(ctx, "cr_attn_paged", args, pages->dtype, pages->kv_heads, pages->head_dim));
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
    CR_TRY(check_heads(ctx, "cr_attn_decode", args, pages->dtype, pages->kv_heads, pages->head_dim));
    if (args->n_tokens != args->n) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: one query token per entry");
    if (n_groups && (!d_group_off || !d_shared)) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: NULL groups");
    if (n_groups > (1u << 24)) return cr_fail(ctx, CR_EINVAL, "cr_attn_decode: %u groups", n_groups);
    if (args->n == 0) return CR_OK;

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
    f.heads = K.heads * F.nsub;
    f.max_cta = 2 * (uint32_t)ctx->num_sms;
    f.min_tiles = kFewMinTiles;
    plan_in g = f;
    g.cu_q = d_group_off;
    g.heads = K.heads;
    g.tok_blk = 2 * R.tq;
    g.max_blk = args->n / g.tok_blk + (n_groups < args->n ? n_groups : args->n);
    g.max_cta = (uint32_t)ctx->num_sms;
    g.min_tiles = kRowsMinTiles;

    const plan_mem mf(f.max_blk, f.max_cta, f.n), mg(g.max_blk, g.max_cta, n_groups);
    void *base;
    CR_TRY(cr_scratch(ctx, SCR_ATTN_PLAN, mf.bytes + mg.bytes, &base));
    mf.point(static_cast<char *>(base), f, F);
    mg.point(static_cast<char *>(base) + mf.bytes, g, R);
    CR_TRY(part_mem(ctx, SCR_ATTN_FEW, F, f.max_cta, 16, D));
    if (n_groups) {
        CR_TRY(part_mem(ctx, SCR_ATTN_PART, R, g.max_cta, 2 * kRowsTile, D));
        const size_t heads = (size_t)args->n * args->q_heads;
        void *p;
        CR_TRY(cr_scratch(ctx, SCR_ATTN_PFX, heads * (D + 1) * 4, &p));
        F.pfx = R.pfx = static_cast<float *>(p);
        F.pfx_lse = R.pfx_lse = F.pfx + heads * D;
        R.to_pfx = 1;
        CR_LAUNCH(ctx, k_attn_plan<PLAN_FEW>, 2, 1024, 0, f, g, ctx->d_status);
        CR_TRY(rows(ctx, R, K, args, g.max_cta));
    } else {
        CR_LAUNCH(ctx, k_attn_plan<PLAN_FEW>, 1, 1024, 0, f, f, ctx->d_status);
    }
    return few(ctx, F, K, f.max_cta);
}
