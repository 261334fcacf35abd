// Rotary positions, writing of new tokens into pages (rotated, in 16 or 8 bits) and reading back
// (include/cacheroute.h).
//
// Angles.  The k-th pair's frequency is held as a 64-bit share of a full turn, so position times frequency is an integer
// product whose overflow drops whole turns: the angle of the furthest position is exact for that share to the 2^-32 turns
// that are used of it (a share is off by 2^-65 turns, the furthest position's product by 2^-34), where a 32-bit product would
// be off by 2^-24 of all the turns made.
//
// All three calls move each element once (2 bytes in, 2 or 1 out) and are bound by that, or by the latency of their
// dependent reads (list, length, table, page) where there are few tokens.  A lane holds V consecutive elements of a
// head: eight, or four where the half layout's pairs are not eights; with that layout its pairs' other elements are
// pairs / V lanes away (shuffles).  Cosines and sines are made once for a CTA's tokens and shared by its heads.
#include <math.h>

#include "cr_attn_index.cuh"
#include "cr_pages.cuh"
#include "cr_tensor.cuh"

namespace {

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kSlice = 32;     // tokens whose cosines and sines a CTA holds
constexpr uint32_t kPairs = 64;     // of a head, at most
constexpr uint32_t kUnits = 4;      // heads that a warp takes at once
constexpr uint32_t kDepth = 3;      // such takes under way
constexpr uint32_t kRing = kWarps * kDepth * kUnits * 512;  // bytes of shared memory for them
constexpr uint32_t kShortList = 1024;

struct rope_in {
    const uint64_t *turn;  // NULL: no rotation
    uint32_t pairs, layout;
    float scale, dir;      // dir: -1 inverse
};

// Cosines and sines of a slice: (s cos, +-s sin) of a token's pairs.  A lane's pairs are E (a power of two) that follow one
// another; the first two of each lane lie together, then the next two: lanes read 16 bytes side by side.
struct rope_shared {
    float4 cs[kSlice * kPairs / 2];
};

// Cosine and sine of t * 2^-32 turns, each within 0.73 units in the last place of a 32-bit number in the first octant: what
// they multiply is rounded to three bits later on, and a cosine that is off by 2^-23 decides one number in a million
// differently.  Whole quarters are dropped as integers; the angle of what is left, |r| <= 2^29, is the sum of th, the
// 32-bit product, and e, what that product lacks; then the Taylor series at th (behind the last term, at pi / 4: 2.3e-9 of
// the angle for the sine, 1.2e-10 for the cosine) and e times the other function.
__device__ __forceinline__ void cos_sin_turn(uint32_t t, float &c, float &s)
{
    constexpr float kHi = 0x1.921fb6p-30f, kLo = -0x1.777a5cp-55f;  // 2 pi * 2^-32
    const uint32_t quarter = (t + (1u << 29)) >> 30;
    const int r = (int)(t - (quarter << 30));
    const float rh = (float)r, rl = (float)(r - (int)rh);
    const float th = rh * kHi, e = fmaf(rh, kHi, -th) + fmaf(rh, kLo, rl * kHi);
    const float z = th * th, zl = fmaf(th, th, -z);
    const float ps = fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6);
    const float sn = th + fmaf(th * z, ps, e * fmaf(-0.5f, z, 1.f));
    const float pc = fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24);
    const float h = fmaf(-0.5f, z, 1.f), hl = fmaf(-0.5f, z, 1.f - h);  // 1 - z / 2, and what that lacks
    const float cs = h + fmaf(z * z, pc, hl + fmaf(-e, th, -0.5f * zl));
    c = quarter & 1 ? sn : cs;
    s = quarter & 1 ? cs : sn;
    if ((quarter + 1) & 2) c = -c;  // quarters 1 and 2
    if (quarter & 2) s = -s;
}

// The slice's cosines and sines; pos(j): position of its j-th token; E: pairs of a lane.
template <typename POS>
__device__ __forceinline__ void make_angles(const rope_in &R, rope_shared &S, uint32_t count, uint32_t E, POS pos)
{
    const uint32_t k = threadIdx.x % kPairs, g = k / E, r = k % E;
    if (k >= R.pairs) return;
    const uint64_t share = R.turn[k];
    float2 *to = reinterpret_cast<float2 *>(S.cs) + ((r >> 1) * (kPairs / E) + g) * 2 + (r & 1);
    for (uint32_t j = threadIdx.x / kPairs; j < count; j += kThreads / kPairs) {
        const uint64_t turn = (uint64_t)(int64_t)pos(j) * share;
        float sn, cs;
        cos_sin_turn((uint32_t)(turn >> 32), cs, sn);
        to[j * kPairs] = make_float2(cs * R.scale, sn * R.scale * R.dir);
    }
}

// V 16-bit elements
template <int V>
struct __align__(2 * V) elems {
    uint32_t w[V / 2];
};
template <bool BF16, int V>
__device__ __forceinline__ void unpack(const elems<V> &v, float *x)
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        if (BF16) {
            x[2 * i] = __uint_as_float(v.w[i] << 16);
            x[2 * i + 1] = __uint_as_float(v.w[i] & 0xffff0000u);
        } else {
            const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&v.w[i]));
            x[2 * i] = a.x;
            x[2 * i + 1] = a.y;
        }
    }
}
template <bool BF16, int V>
__device__ __forceinline__ elems<V> pack(const float *x)
{
    elems<V> v;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) v.w[i] = cr_pack16<BF16>(x[2 * i], x[2 * i + 1]);
    return v;
}

// A lane's place in a token's head, elements d .. d+V-1, and what rotates them.
template <bool BF16, int V>
struct lane_rope {
    uint32_t d, sub, per;  // sub: of which of the warp's `per` tokens
    int from;              // half layout: lane with the pairs' other elements
    bool on, turns, half;
    float c[V], s[V];      // what multiplies the lane's own elements, and their partners
    __device__ __forceinline__ lane_rope(uint32_t head_dim, const rope_in &R)
    {
        const uint32_t lane = threadIdx.x & 31, lanes = (head_dim <= 64 ? 64 : 128) / V, l = lane & (lanes - 1);
        per = 32 / lanes;
        sub = lane / lanes;
        d = V * l;
        on = d < head_dim;
        turns = R.turn && d < 2 * R.pairs;
        half = R.layout == CR_ROTARY_HALF;
        from = (int)lane;
        if (turns && half) from = d >= R.pairs ? (int)(lane - R.pairs / V) : (int)(lane + R.pairs / V);
    }
    // of the slice's j-th token
    __device__ __forceinline__ void load(const rope_in &R, const rope_shared &S, uint32_t j)
    {
        if (!turns) return;
        if (half) {
            const bool second = d >= R.pairs;
            const float4 *p = S.cs + j * (kPairs / 2) + (second ? d - R.pairs : d) / V;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float4 a = p[i * (kPairs / V)];
                c[2 * i] = a.x, c[2 * i + 1] = a.z;
                s[2 * i] = second ? a.y : -a.y, s[2 * i + 1] = second ? a.w : -a.w;
            }
        } else {
            const float4 *p = S.cs + j * (kPairs / 2) + d / V;
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const float4 a = p[i * (2 * kPairs / V)];
                c[4 * i] = c[4 * i + 1] = a.x;
                c[4 * i + 2] = c[4 * i + 3] = a.z;
                s[4 * i] = -a.y, s[4 * i + 1] = a.y;
                s[4 * i + 2] = -a.w, s[4 * i + 3] = a.w;
            }
        }
    }
    // The whole warp calls it.  Elements that are not rotated are given back as they are.
    __device__ __forceinline__ void rotate(const rope_in &R, const elems<V> &v, float *x) const
    {
        unpack<BF16, V>(v, x);
        if (!R.turn) return;
        float y[V];
        if (half) {
            elems<V> o;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) o.w[i] = __shfl_sync(~0u, v.w[i], from);
            unpack<BF16, V>(o, y);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = x[i ^ 1];
        }
        if (turns) {
#pragma unroll
            for (int i = 0; i < V; i += 2)
                cr_unpair(cr_fma2(cr_pair(x[i], x[i + 1]), cr_pair(c[i], c[i + 1]), cr_mul2(cr_pair(y[i], y[i + 1]), cr_pair(s[i], s[i + 1]))),
                          x[i], x[i + 1]);
        }
    }
};

// V elements to shared memory and from there; the thread that has copied them takes them.
template <int V>
__device__ __forceinline__ void copy_async(uint32_t dst, const uint16_t *src)
{
    if (V == 8)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
template <int V>
__device__ __forceinline__ elems<V> take(uint32_t at)
{
    elems<V> v;
    if (V == 8)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[V / 2 - 2]), "=r"(v.w[V / 2 - 1])
                     : "r"(at)
                     : "memory");
    else
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "r"(at) : "memory");
    return v;
}

// A CTA's tokens, the first count of the slice, and its n heads: few of them are shared out over all warps.  A warp has
// kDepth takes of up to kUnits heads under way, in its part of the ring; ready() makes the angles meanwhile.
template <bool BF16, int V, typename READY>
__device__ __forceinline__ void move_heads(lane_rope<BF16, V> &L, const rope_in &R, const rope_shared &S, uint32_t ring, uint32_t count,
                                           uint32_t n, bool lost, const uint16_t *src, uint64_t src_token, uint64_t src_head, uint16_t *dst,
                                           uint64_t dst_token, uint64_t dst_head, READY ready)
{
    const uint32_t rounds = (count + L.per - 1) / L.per, each = max(1u, min(kUnits, n * rounds / kWarps));
    const uint32_t tasks = rounds * ((n + each - 1) / each);
    const uint32_t mine = ring + (threadIdx.x >> 5) * (kDepth * kUnits * 512) + (threadIdx.x & 31) * (2 * V);
    auto issue = [&](uint32_t task, uint32_t slot) {
        if (task < tasks) {
            const uint32_t g = task / rounds, j = (task - g * rounds) * L.per + L.sub, heads = min(each, n - g * each);
            const uint16_t *at = src + (uint64_t)j * src_token + g * each * src_head + L.d;
            if (L.on && j < count)
                for (uint32_t u = 0; u < heads; ++u, at += src_head) copy_async<V>(mine + (slot * kUnits + u) * 512, at);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    uint32_t task = threadIdx.x >> 5, slot = 0, loaded = ~0u;
#pragma unroll
    for (uint32_t i = 0; i < kDepth; ++i) issue(task + i * kWarps, i);
    ready();
    for (; task < tasks; task += kWarps) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        const uint32_t g = task / rounds, i = task - g * rounds, j = i * L.per + L.sub, heads = min(each, n - g * each);
        if (i != loaded) L.load(R, S, min(j, count - 1));
        loaded = i;
        uint16_t *at = dst + (uint64_t)j * dst_token + g * each * dst_head + L.d;
        const bool in = L.on && j < count;
#pragma unroll 4
        for (uint32_t u = 0; u < heads; ++u, at += dst_head) {
            elems<V> v = take<V>(mine + (slot * kUnits + u) * 512);
            if (R.turn) {
                float x[V];
                L.rotate(R, v, x);
                if (L.turns) v = pack<BF16, V>(x);
            }
            if (lost) {
#pragma unroll
                for (int e = 0; e < V / 2; ++e) v.w[e] = 0;
            }
            if (in) *reinterpret_cast<elems<V> *>(at) = v;
        }
        issue(task + kDepth * kWarps, slot);
        slot = slot + 1 == kDepth ? 0 : slot + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// ---- 8-bit numbers -----------------------------------------------------------------------------
// Exponents of a block's power, and what rounds to an infinity in the 16-bit type.
template <bool BF16>
struct e4m3_range {
    static constexpr int kMin = BF16 ? -100 : -15, kMax = BF16 ? 120 : 8;
    static constexpr float kInf = BF16 ? 0x1.ffp127f : 65520.f;
};
// The smallest 2^e for which 448 * 2^e = 1.75 * 2^(e+8) reaches `top`.
template <bool BF16>
__device__ __forceinline__ float block_power(float top)
{
    const uint32_t b = __float_as_uint(top);
    int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
    e = max(e4m3_range<BF16>::kMin, min(e4m3_range<BF16>::kMax, e));
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
// V e4m3 numbers of x in units of a block's power, 1 / by; big: some may be no finite numbers of the 16-bit type, or the
// power is the largest (numbers up to 240).
template <bool BF16, int V>
__device__ __forceinline__ void to_e4m3(const float *x, float by, float most, bool big, uint32_t *q)
{
    float y[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) cr_unpair(cr_mul2(cr_pair(x[i], x[i + 1]), cr_pair(by, by)), y[i], y[i + 1]);
    if (big) {
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fabsf(x[i]) < e4m3_range<BF16>::kInf ? fminf(fmaxf(y[i], -most), most) : __int_as_float(0x7fffffff);
    }
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y[4 * i + 1]), "f"(y[4 * i]));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y[4 * i + 3]), "f"(y[4 * i + 2]));
        q[i] = (uint32_t)lo | (uint32_t)hi << 16;
    }
}
__device__ __forceinline__ void unpack_e4m3(uint32_t v, float *x)
{
    uint32_t a, b;
    cr_e4m3_halves(v, a, b);
    const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&a)), q = __half22float2(*reinterpret_cast<const __half2 *>(&b));
    x[0] = p.x, x[1] = p.y, x[2] = q.x, x[3] = q.y;
}

// ---- rotating packed tokens ----------------------------------------------------------------------
struct rope_tokens {
    const uint16_t *x;
    uint16_t *o;
    uint64_t x_token, x_head, o_token, o_head;
    const int32_t *pos;
    uint32_t n_tokens, heads, head_dim;
};

// blockIdx.x: `tokens` of them; blockIdx.y: a share of the heads.  Bound by HBM: 26,000 tokens of 28 heads of 128, 64 of
// them in pairs, 58 us, 6.5 TB/s.
template <bool BF16, int V>
__global__ void __launch_bounds__(kThreads) k_rope(const __grid_constant__ rope_tokens A, const __grid_constant__ rope_in R, uint32_t tokens)
{
    __shared__ __align__(16) rope_shared S;
    extern __shared__ __align__(16) uint32_t dyn[];
    cr_launch_next();
    cr_wait_previous();
    const uint32_t t0 = blockIdx.x * tokens, count = min(tokens, A.n_tokens - t0);
    lane_rope<BF16, V> L(A.head_dim, R);
    const uint32_t h0 = (uint32_t)((uint64_t)A.heads * blockIdx.y / gridDim.y),
                   h1 = (uint32_t)((uint64_t)A.heads * (blockIdx.y + 1) / gridDim.y);
    move_heads(L, R, S, cr_smem(dyn), count, h1 - h0, false, A.x + (uint64_t)t0 * A.x_token + h0 * A.x_head, A.x_token, A.x_head,
               A.o + (uint64_t)t0 * A.o_token + h0 * A.o_head, A.o_token, A.o_head, [&] {
                   make_angles(R, S, count, L.half ? V : V / 2, [&](uint32_t j) { return A.pos[t0 + j]; });
                   __syncthreads();
               });
}

// ---- writing into pages ----------------------------------------------------------------------------
struct append_in {
    const uint16_t *q, *k, *v;
    uint16_t *qo;
    uint64_t q_token, q_head, o_token, o_head, k_token, k_head, v_token, v_head;
    const int32_t *cu, *seqs;
    const int32_t *claim;  // long lists: the first entry of each row that has tokens
    uint32_t n, n_tokens, q_heads, step_log2;  // step: positions of a slot
    uint32_t kv_split;     // blockIdx.y below: a share of the key heads, the others one of the query heads
};

__global__ void __launch_bounds__(256) k_claim_clear(int32_t *claim, const int32_t *seqs, uint32_t n, uint32_t n_seqs)
{
    cr_launch_next();
    cr_wait_previous();
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const int row = seqs[i];
        if (row >= 0 && (uint32_t)row < n_seqs) claim[row] = 0x7fffffff;
    }
}
__global__ void __launch_bounds__(256) k_claim(int32_t *claim, const int32_t *seqs, const int32_t *cu, uint32_t n, uint32_t n_seqs)
{
    cr_launch_next();
    cr_wait_previous();
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const int row = seqs[i];
        if (row >= 0 && (uint32_t)row < n_seqs && cu[i] < cu[i + 1]) atomicMin(claim + row, (int)i);
    }
}

// What a CTA works on: up to `step` consecutive positions of a row, all in one block of a page.
struct slot_work {
    int t0, pos, count;     // first token, its position (the entry's first: 0, where there is no row), tokens
    int row;
    uint32_t entry;
    uint32_t place;         // of the first token in its page
    bool lost;              // the positions are outside the row
};
// The slot of this CTA belongs to the last entry whose slots begin at or before it.  Every warp looks for itself.
// What it finds is what reading the tokens takes; their page (page_of_slot) is found while they are on their way.
__device__ __forceinline__ bool find_slot(const pages_in &P, const append_in &A, slot_work &W)
{
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t s = blockIdx.x;
    uint32_t lo = 0, span = A.n;
    while (span > 1) {
        const uint32_t step = (span + 31) / 32, i = lo + lane * step;
        const bool in = lane * step < span && cr_slot_of(max(A.cu[i], 0), i, A.step_log2) <= s;
        const uint32_t some = __ballot_sync(~0u, in), last = some ? 31 - __clz(some) : 0;
        lo += last * step;
        span = min(step, span - last * step);
    }
    W.entry = lo;
    const int a = min(max(A.cu[lo], 0), (int)A.n_tokens), b = min(max(A.cu[lo + 1], a), (int)A.n_tokens);
    const uint64_t mine = cr_slot_of(a, lo, A.step_log2);
    if (s < mine) return false;
    const int row = A.seqs ? A.seqs[lo] : (int)lo;
    const bool have = row >= 0 && (uint32_t)row < P.n_seqs;
    const int len = have ? P.lens[row] : b - a;
    const cr_positions at = cr_slot_positions(len, b - a, s - mine, A.step_log2);
    if (at.begin >= at.end) return false;
    W.t0 = b - (int)(len - at.begin);
    W.pos = (int)at.begin;
    W.count = (int)(at.end - at.begin);
    W.row = row;
    W.place = (uint32_t)at.begin & (P.page - 1);
    W.lost = !have || at.begin < 0 || (uint64_t)at.begin >> P.page_log2 >= P.max_pages;
    return true;
}
// The page of a slot's tokens, or -1: their keys and values go nowhere.  The whole CTA calls it.
__device__ __forceinline__ int page_of_slot(const pages_in &P, const append_in &A, const slot_work &W)
{
    int page = -1;
    if (!W.lost) {
        const int p = P.table[(uint64_t)W.row * P.max_pages + ((uint32_t)W.pos >> P.page_log2)];
        // pages that other rows name are not this row's to write (k_kv_write)
        if (p >= 0 && (uint32_t)p < P.n_pages && P.ref[p] <= 1) page = p;
        if (A.claim && A.claim[W.row] != (int)W.entry) page = -1;
    }
    if (A.seqs && !A.claim) {  // a row that an entry before this one names is that one's, if it has tokens
        bool twice = false;
        for (uint32_t i = threadIdx.x; i < W.entry; i += kThreads) twice |= A.seqs[i] == W.row && A.cu[i] < A.cu[i + 1];
        if (__syncthreads_or(twice)) page = -1;
    }
    if (page < 0 && threadIdx.x == 0) atomicOr(P.status, CR_FLAG_BADPAGES);
    return page;
}

// Bound by its instructions: 12 prompts of 1 to 4,096 tokens, 28/4 heads of 128, 8 bits, 110 us with issue slots 71% busy
// (the bytes alone: 73 us).  Keys and values in registers until their power is known, instead of in shared memory: 166.
template <bool BF16, bool E4M3, int V>
__global__ void __launch_bounds__(kThreads, 3) k_kv_append(const __grid_constant__ pages_in P, const __grid_constant__ append_in A,
                                                        const __grid_constant__ rope_in R, uint32_t layer)
{
    __shared__ __align__(16) rope_shared S;
    extern __shared__ __align__(16) uint32_t dyn[];
    cr_launch_next();
    cr_wait_previous();
    slot_work W;
    if (!find_slot(P, A, W)) return;
    const uint32_t warp = threadIdx.x >> 5, count = (uint32_t)W.count;
    lane_rope<BF16, V> L(P.head_dim, R);
    auto angles = [&](uint32_t s0, uint32_t n) {
        __syncthreads();
        if (R.turn) make_angles(R, S, n, L.half ? V : V / 2, [&](uint32_t j) { return W.pos + (int)(s0 + j); });
        __syncthreads();
    };
    if (blockIdx.y >= A.kv_split) {  // a share of the query heads
        const uint32_t y = blockIdx.y - A.kv_split, ny = gridDim.y - A.kv_split;
        const uint32_t q0 = (uint32_t)((uint64_t)A.q_heads * y / ny), q1 = (uint32_t)((uint64_t)A.q_heads * (y + 1) / ny);
        for (uint32_t s0 = 0; s0 < count; s0 += kSlice) {
            const uint32_t n = min(kSlice, count - s0);
            const uint64_t t = (uint32_t)W.t0 + s0;
            move_heads(L, R, S, cr_smem(dyn), n, q1 - q0, W.lost, A.q + t * A.q_token + q0 * A.q_head, A.q_token, A.q_head,
                       A.qo + t * A.o_token + q0 * A.o_head, A.o_token, A.o_head, [&] { angles(s0, n); });
        }
        return;
    }
    const uint32_t y = blockIdx.y, ny = A.kv_split;  // a share of the key heads
    const uint32_t k0 = (uint32_t)((uint64_t)P.kv_heads * y / ny), nk = (uint32_t)((uint64_t)P.kv_heads * (y + 1) / ny) - k0;
    if (!E4M3) {
        const int page = page_of_slot(P, A, W);
        if (page < 0) return;
        uint8_t *kd = P.plane(2 * layer) + 2 * (page * P.page_stride), *vd = P.plane(2 * layer + 1) + 2 * (page * P.page_stride);
        for (uint32_t s0 = 0; s0 < count; s0 += kSlice) {
            const uint32_t n = min(kSlice, count - s0);
            const uint64_t t = (uint32_t)W.t0 + s0;
            const uint64_t to = (uint64_t)(W.place + s0) * P.token_stride + k0 * P.head_stride;
            move_heads(L, R, S, cr_smem(dyn), n, nk, false, A.k + t * A.k_token + k0 * A.k_head, A.k_token, A.k_head,
                       reinterpret_cast<uint16_t *>(kd) + to, P.token_stride, P.head_stride, [&] { angles(s0, n); });
            move_heads(L, rope_in{}, S, cr_smem(dyn), n, nk, false, A.v + t * A.v_token + k0 * A.v_head, A.v_token, A.v_head,
                       reinterpret_cast<uint16_t *>(vd) + to, P.token_stride, P.head_stride, [] {});
        }
        return;
    }

    // 8 bits.  The slice's keys and values lie in shared memory, head by head (keys' first), each row of a token's
    // elements together, until their powers are known.  A warp has a head, or a share of its tokens where heads are few.
    uint32_t *top = dyn;                                                    // [2 nk] largest magnitudes, then powers
    float *power = reinterpret_cast<float *>(dyn);                          // [2 nk], then [2 nk] old over new
    uint32_t *odd = dyn + 4 * nk;                                           // [2 nk] some are no finite numbers
    const uint32_t row = P.head_dim * 2, bytes = row * min(kSlice, 1u << A.step_log2);  // of a token, of a head
    const uint32_t rows = (cr_smem(odd + 2 * nk) + 15u) & ~15u;
    for (uint32_t i = threadIdx.x; i < 2 * nk; i += kThreads) top[i] = odd[i] = 0;
    auto fetch = [&](uint32_t s0, uint32_t n) {
        for (uint32_t g = warp; g < 2 * nk; g += kWarps) {
            const bool key = g < nk;
            const uint64_t token = key ? A.k_token : A.v_token;
            const uint16_t *src = (key ? A.k + (k0 + g) * A.k_head : A.v + (k0 + g - nk) * A.v_head) + ((uint32_t)W.t0 + s0 + L.sub) * token + L.d;
            uint32_t to = rows + g * bytes + L.sub * row + L.d * 2;
            if (L.on)
                for (uint32_t j = L.sub; j < n; j += L.per, src += L.per * token, to += L.per * row) copy_async<V>(to, src);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto fetched = [&]() {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
    };
    // use(head, behind nk: a value's; token of the slice; numbers) for the share of heads and tokens that this warp has;
    // end(head) behind each head
    const uint32_t parts = max(1u, kWarps / (2 * nk));
    auto each = [&](uint32_t n, auto use, auto end) {
        const uint32_t rounds = (n + L.per - 1) / L.per;
        for (uint32_t w = warp; w < 2 * nk * parts; w += kWarps) {
            const uint32_t g = w / parts;
            for (uint32_t i = w - g * parts; i < rounds; i += parts) {
                const uint32_t j = min(i * L.per + L.sub, n - 1);  // the last token stands for those behind
                float x[V];
                const elems<V> v = L.on ? take<V>(rows + g * bytes + j * row + L.d * 2) : elems<V>{};
                if (g < nk) {
                    L.load(R, S, j);
                    L.rotate(R, v, x);
                } else {
                    unpack<BF16, V>(v, x);
                }
                use(g, i * L.per + L.sub, x);
            }
            end(g);
        }
    };
    float m = 0.f;  // the largest of a head's
    auto measure = [&](uint32_t n) {
        each(
            n,
            [&](uint32_t g, uint32_t, const float *x) {
                float mine = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) mine = fmaxf(mine, fabsf(x[e]));
                if (mine >= e4m3_range<BF16>::kInf) {
                    mine = 0.f;
#pragma unroll
                    for (int e = 0; e < V; ++e) mine = fabsf(x[e]) < e4m3_range<BF16>::kInf ? fmaxf(mine, fabsf(x[e])) : mine;
                    odd[g] = 1;
                }
                m = fmaxf(m, mine);
            },
            [&](uint32_t g) {
                const uint32_t all = __reduce_max_sync(~0u, __float_as_uint(m));
                if ((threadIdx.x & 31) == 0) atomicMax(top + g, all);
                m = 0.f;
            });
    };
    uint32_t last = 0;  // the slice that is there
    int page = -1;
    for (uint32_t s0 = 0; s0 < count; s0 += kSlice) {
        const uint32_t n = min(kSlice, count - s0);
        if (s0) __syncthreads();
        fetch(s0, n);
        if (s0 == 0) {
            page = page_of_slot(P, A, W);
            if (page < 0) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                return;
            }
        }
        angles(s0, n);
        fetched();
        measure(n);
        last = s0;
    }

    // the blocks' powers
    uint8_t *kd = P.plane(2 * layer) + page * P.page_stride, *vd = P.plane(2 * layer + 1) + page * P.page_stride;
    constexpr float kTop = BF16 ? 0x1p120f : 0x1p8f;  // the largest one
    __syncthreads();
    const uint32_t nb_log2 = P.page_log2 - P.block_log2, block = W.place >> P.block_log2, before = W.place & ((1u << P.block_log2) - 1);
    for (uint32_t i = threadIdx.x; i < 2 * nk; i += kThreads) {
        const uint32_t h = k0 + (i < nk ? i : i - nk);
        float *at = P.scales(2 * layer + (i >= nk), (uint32_t)page) + (h << nb_log2) + block;
        float now = block_power<BF16>(__uint_as_float(top[i]));
        float ratio = 1.f;
        if (before) {
            const float old = *at;  // a power of two in the type's range: what is none becomes one
            now = fmaxf(now, fminf(__uint_as_float(__float_as_uint(old) & 0x7f800000u), kTop));
            ratio = old / now;
        }
        *at = now;
        power[i] = now;
        power[2 * nk + i] = ratio;
    }
    __syncthreads();
    // the tokens that were there, where the power has grown
    for (uint32_t i = before ? warp : 2 * nk; i < 2 * nk; i += kWarps) {
        const float ratio = power[2 * nk + i];
        if (ratio == 1.f) continue;
        const uint32_t h = k0 + (i < nk ? i : i - nk);
        uint8_t *base = (i < nk ? kd : vd) + h * P.head_stride + L.d;
        for (uint32_t j = L.sub; j < before; j += L.per) {
            if (!L.on) continue;
            uint32_t *at = reinterpret_cast<uint32_t *>(base + (uint64_t)(W.place - before + j) * P.token_stride);
#pragma unroll
            for (int e = 0; e < V / 4; ++e) {
                float z[4];
                unpack_e4m3(at[e], z);
                to_e4m3<BF16, 4>(z, ratio, 448.f, false, at + e);
            }
        }
    }
    for (uint32_t s0 = last;; s0 -= kSlice) {  // from the last slice, which is there, to the first
        const uint32_t n = min(kSlice, count - s0);
        if (s0 != last) {
            __syncthreads();
            fetch(s0, n);
            angles(s0, n);
            fetched();
        }
        each(
            n,
            [&](uint32_t g, uint32_t j, const float *x) {
                const float p = power[g];
                uint32_t q[V / 4];
                to_e4m3<BF16, V>(x, __uint_as_float((254u << 23) - __float_as_uint(p)), p >= kTop ? 240.f : 448.f, p >= kTop || odd[g], q);
                if (!L.on || j >= n) return;
                const uint32_t h = k0 + (g < nk ? g : g - nk);
                uint8_t *to = (g < nk ? kd : vd) + (uint64_t)(W.place + s0 + j) * P.token_stride + h * P.head_stride + L.d;
                if (V == 8)
                    *reinterpret_cast<uint2 *>(to) = make_uint2(q[0], q[V / 4 - 1]);
                else
                    *reinterpret_cast<uint32_t *>(to) = q[0];
            },
            [](uint32_t) {});
        if (s0 == 0) break;
    }
}

// ---- reading back ----------------------------------------------------------------------------------
struct read_in {
    uint16_t *k, *v;
    uint64_t k_token, k_head, v_token, v_head;
    const int32_t *cu, *seqs, *start;
    uint32_t n, n_tokens;
};

// A CTA takes kReadTokens tokens.  A lane each finds where they lie (list, length, table: a chain of reads), then they are
// copied, V elements a lane, two reads of keys and two of values under way.  (CTAs that take one piece after the other and
// look the next one up meanwhile: 71 -> 80 us for 130,000 tokens of 8 heads of 64.)  Those take 72 us, 5.7 TB/s.
constexpr uint32_t kReadTokens = 32;
template <bool BF16, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_kv_read(const __grid_constant__ pages_in P, const __grid_constant__ read_in A, uint32_t layer)
{
    constexpr int V = E4M3 ? 16 : 8;
    __shared__ uint2 at[kReadTokens];  // page (none: ~0), place in it
    cr_launch_next();
    cr_wait_previous();
    const uint32_t t0 = blockIdx.x * kReadTokens, count = min(kReadTokens, A.n_tokens - t0);
    if (threadIdx.x < count) {
        const int t = (int)(t0 + threadIdx.x);
        uint32_t lo = 0, hi = A.n;  // last entry that begins at or before t
        while (hi - lo > 1) {
            const uint32_t m = (lo + hi) >> 1;
            if (A.cu[m] <= t)
                lo = m;
            else
                hi = m;
        }
        const int a = A.n ? A.cu[lo] : 0, b = A.n ? A.cu[lo + 1] : 0;
        uint2 w = make_uint2(~0u, 0);
        if (a <= t && t < b) {
            const int row = A.seqs ? A.seqs[lo] : (int)lo;
            if (row >= 0 && (uint32_t)row < P.n_seqs) {
                const int len = P.lens[row];
                const long long pos = (A.start ? (long long)A.start[lo] : (long long)len - ((long long)b - a)) + (t - a);
                if (pos >= 0 && pos < len && ((uint64_t)pos >> P.page_log2) < P.max_pages) {
                    const int p = P.table[(uint64_t)row * P.max_pages + (uint32_t)(pos >> P.page_log2)];
                    if (p >= 0 && (uint32_t)p < P.n_pages) w = make_uint2((uint32_t)p, (uint32_t)pos & (P.page - 1));
                }
            }
        }
        if (w.x == ~0u) atomicOr(P.status, CR_FLAG_BADPAGES);
        at[threadIdx.x] = w;
    }
    __syncthreads();
    const uint32_t per = (P.head_dim + V - 1) / V, words = P.kv_heads * per, nb_log2 = P.page_log2 - P.block_log2;
    const uint8_t *kp = P.plane(2 * layer), *vp = P.plane(2 * layer + 1);
    // the tokens' words one after the other, two at a time in each lane
    const uint32_t total = count * words;
    for (uint32_t i0 = threadIdx.x; i0 < total; i0 += 2 * kThreads) {
        uint4 in[2][2];
        float f[2][2];
        uint32_t j[2], h[2], d[2];
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e) {
            const uint32_t i = i0 + e * kThreads;
            j[e] = i / words;
            h[e] = (i - j[e] * words) / per;
            d[e] = (i - j[e] * words - h[e] * per) * V;
            const uint2 w = i < total ? at[j[e]] : make_uint2(~0u, 0);
            const uint64_t off = (w.x * P.page_stride + w.y * P.token_stride + h[e] * P.head_stride + d[e]) << P.size_log2;
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c) {
                in[e][c] = make_uint4(0, 0, 0, 0);
                f[e][c] = 0.f;
                if (w.x == ~0u) continue;
                in[e][c] = *reinterpret_cast<const uint4 *>((c ? vp : kp) + off);
                if (E4M3) f[e][c] = P.scales(2 * layer + c, w.x)[(h[e] << nb_log2) + (w.y >> P.block_log2)];
            }
        }
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e) {
            if (i0 + e * kThreads >= total) continue;
            const uint64_t t = t0 + j[e];
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c) {
                uint4 *dst = reinterpret_cast<uint4 *>(c ? A.v + t * A.v_token + h[e] * A.v_head + d[e] : A.k + t * A.k_token + h[e] * A.k_head + d[e]);
                if (E4M3) {
                    const uint32_t q[4] = {in[e][c].x, in[e][c].y, in[e][c].z, in[e][c].w};
                    uint32_t o[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float x[4];
                        unpack_e4m3(q[k], x);
                        o[2 * k] = cr_pack16<BF16>(x[0] * f[e][c], x[1] * f[e][c]);
                        o[2 * k + 1] = cr_pack16<BF16>(x[2] * f[e][c], x[3] * f[e][c]);
                    }
                    dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
                    dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
                } else {
                    dst[0] = in[e][c];
                }
            }
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------
int rotary_check(cr_ctx *ctx, const char *who, const cr_rotary *r, uint32_t head_dim, rope_in &R)
{
    R = rope_in{};
    if (!r) return CR_OK;
    if (!r->d_turn || ((uintptr_t)r->d_turn & 7)) return cr_fail(ctx, CR_EINVAL, "%s: d_turn must hold the pairs' frequencies", who);
    if (!r->pairs || (r->pairs & 3) || 2 * (uint64_t)r->pairs > head_dim)
        return cr_fail(ctx, CR_EINVAL, "%s: %u rotated pairs in heads of %u: a multiple of 4, at most half a head", who, r->pairs, head_dim);
    if (r->layout > CR_ROTARY_PAIRS) return cr_fail(ctx, CR_EINVAL, "%s: rotary layout %u", who, r->layout);
    if (!(fabsf(r->scale) <= 3.402823466e38f)) return cr_fail(ctx, CR_EINVAL, "%s: rotary scale must be finite", who);
    R.turn = r->d_turn;
    R.pairs = r->pairs;
    R.layout = r->layout;
    R.scale = r->scale;
    R.dir = r->inverse ? -1.f : 1.f;
    return CR_OK;
}

// A launch whose kernel may take up to kMostSmem bytes of dynamic shared memory.
constexpr size_t kMostSmem = 52 * 1024;
template <auto KERN, typename... T>
int launch(cr_ctx *ctx, const char *what, dim3 grid, size_t smem, const T &...args)
{
    static_assert(kRing <= kMostSmem, "shared memory of a CTA");
    static unsigned long long raised = 0;  // devices
    const unsigned long long bit = 1ull << (ctx->device & 63);
    if (!(raised & bit)) {
        CR_CUDA(ctx, cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
        raised |= bit;
    }
    return cr_launch_early(ctx, what, KERN, grid, kThreads, smem, args...);
}

// Whether lanes may hold eight elements: the half layout's pairs are then whole lanes apart.
bool by_eight(const rope_in &R) { return !R.turn || R.layout == CR_ROTARY_PAIRS || R.pairs % 8 == 0; }

bool aligned(const void *p, uint64_t a, uint64_t b) { return ((uintptr_t)p & 15) == 0 && (a & 7) == 0 && (b & 7) == 0; }

}  // namespace

extern "C" int cr_rope(cr_ctx *ctx, const cr_rotary *rotary, const cr_rope_args *a)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_rope");
    if (!rotary || !a) return cr_fail(ctx, CR_EINVAL, "cr_rope: NULL rotary or args");
    const uint32_t n_tokens = a->n_tokens, heads = a->heads, head_dim = a->head_dim;
    if (a->dtype > CR_DTYPE_FP16) return cr_fail(ctx, CR_EINVAL, "cr_rope: dtype %u", a->dtype);
    if (!head_dim || head_dim > 128 || (head_dim & 7)) return cr_fail(ctx, CR_EINVAL, "cr_rope: head_dim %u: a multiple of 8, 8..128", head_dim);
    rope_in R;
    CR_TRY(rotary_check(ctx, "cr_rope", rotary, head_dim, R));
    if (n_tokens > (1u << 30) || heads > (1u << 20)) return cr_fail(ctx, CR_EINVAL, "cr_rope: too many tokens or heads");
    if (!n_tokens || !heads) return CR_OK;
    if (!a->d_x || !a->d_out || !a->d_pos) return cr_fail(ctx, CR_EINVAL, "cr_rope: NULL pointer");
    if (!aligned(a->d_x, a->x_token, a->x_head) || !aligned(a->d_out, a->o_token, a->o_head))
        return cr_fail(ctx, CR_EINVAL, "cr_rope: tensors must be 16-byte aligned, strides multiples of 8");
    if (a->d_x == a->d_out && (a->x_token != a->o_token || a->x_head != a->o_head))
        return cr_fail(ctx, CR_EINVAL, "cr_rope: in place, the strides must be the same");
    const rope_tokens A = {static_cast<const uint16_t *>(a->d_x), static_cast<uint16_t *>(a->d_out), a->x_token, a->x_head, a->o_token,
                           a->o_head, a->d_pos, n_tokens, heads, head_dim};
    // 16 tokens share a CTA's beginning, fewer where heads are many.  Few tokens: several CTAs share their heads.
    const uint32_t per = by_eight(R) ? (head_dim <= 64 ? 4 : 2) : (head_dim <= 64 ? 2 : 1);
    const uint32_t tokens = max(per, min(16u, 8 * kWarps * kUnits * per / heads)), blocks = (n_tokens + tokens - 1) / tokens;
    const uint32_t split = max(1u, min((heads + kUnits - 1) / kUnits, 4 * (uint32_t)ctx->num_sms / blocks));
    const dim3 grid(blocks, split);
    const bool bf16 = a->dtype == CR_DTYPE_BF16;
    if (by_eight(R))
        return bf16 ? launch<k_rope<true, 8>>(ctx, "k_rope", grid, kRing, A, R, tokens) : launch<k_rope<false, 8>>(ctx, "k_rope", grid, kRing, A, R, tokens);
    return bf16 ? launch<k_rope<true, 4>>(ctx, "k_rope", grid, kRing, A, R, tokens) : launch<k_rope<false, 4>>(ctx, "k_rope", grid, kRing, A, R, tokens);
}

template <bool BF16, bool E4M3>
static int launch_append(cr_ctx *ctx, dim3 grid, size_t smem, const pages_in &P, const append_in &A, const rope_in &R, uint32_t layer)
{
    return by_eight(R) ? launch<k_kv_append<BF16, E4M3, 8>>(ctx, "k_kv_append", grid, smem, P, A, R, layer)
                       : launch<k_kv_append<BF16, E4M3, 4>>(ctx, "k_kv_append", grid, smem, P, A, R, layer);
}

int cr_append(cr_ctx *ctx, const char *who, const cr_kv_pages *pg, uint32_t layer, const cr_rotary *rotary, const cr_append_args *a)
{
    rope_in R;
    CR_TRY(rotary_check(ctx, who, rotary, pg->head_dim, R));
    const pages_in P = cr_pages_input(ctx, pg);
    append_in A = {};
    A.q = static_cast<const uint16_t *>(a->d_q);
    A.k = static_cast<const uint16_t *>(a->d_k);
    A.v = static_cast<const uint16_t *>(a->d_v);
    A.qo = static_cast<uint16_t *>(a->d_q_out);
    A.q_token = a->q_token;
    A.q_head = a->q_head;
    A.o_token = a->o_token;
    A.o_head = a->o_head;
    A.k_token = a->k_token;
    A.k_head = a->k_head;
    A.v_token = a->v_token;
    A.v_head = a->v_head;
    A.cu = a->d_cu;
    A.seqs = a->d_seqs;
    A.n = a->n;
    A.n_tokens = a->n_tokens;
    A.q_heads = a->q_heads;
    const bool e4m3 = cr_in_8bit(pg->dtype);
    A.step_log2 = e4m3 ? P.block_log2 : (P.page_log2 < 4 ? P.page_log2 : 4);
    if (A.seqs && A.n > kShortList) {  // looking through the list once for every slot would be too long
        void *p;
        CR_TRY(cr_scratch(ctx, SCR_KV_CLAIM, 4 * (size_t)pg->n_seqs, &p));
        int32_t *claim = static_cast<int32_t *>(p);
        const uint32_t blocks = cr_blocks(A.n, 256, 2 * ctx->num_sms);
        CR_TRY(cr_launch_early(ctx, "k_claim_clear", k_claim_clear, dim3(blocks), 256, 0, claim, A.seqs, A.n, P.n_seqs));
        CR_TRY(cr_launch_early(ctx, "k_claim", k_claim, dim3(blocks), 256, 0, claim, A.seqs, A.cu, A.n, P.n_seqs));
        A.claim = claim;
    }
    // Shares of the heads.  8 bits: as many key heads as 48 KB of shared memory hold for a slice (three CTAs an SM);
    // queries: one head a warp at least.
    const uint64_t slots = ((uint64_t)A.n_tokens >> A.step_log2) + 2ull * A.n;
    const uint32_t want = 1 + (uint32_t)(4ull * (uint32_t)ctx->num_sms / slots);
    const uint32_t head = 4 * pg->head_dim * min(kSlice, 1u << A.step_log2), fit = 48 * 1024 / head;
    A.kv_split = min(pg->kv_heads, max(want, e4m3 ? (pg->kv_heads + fit - 1) / fit : 1u));
    const uint32_t q_split = A.q_heads ? min((A.q_heads + kWarps - 1) / kWarps, want) : 0;
    const dim3 grid((uint32_t)slots, A.kv_split + q_split);
    const uint32_t most = (pg->kv_heads + A.kv_split - 1) / A.kv_split;
    const size_t bytes = max((size_t)kRing, e4m3 ? (24 + head) * (size_t)most + 16 : 0);
    if (cr_is_bf16(pg->dtype))
        return e4m3 ? launch_append<true, true>(ctx, grid, bytes, P, A, R, layer) : launch_append<true, false>(ctx, grid, bytes, P, A, R, layer);
    return e4m3 ? launch_append<false, true>(ctx, grid, bytes, P, A, R, layer) : launch_append<false, false>(ctx, grid, bytes, P, A, R, layer);
}

extern "C" int cr_kv_append(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, const cr_rotary *rotary,
                            const cr_append_args *a)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_kv_append");
    CR_TRY(cr_pages_check(ctx, "cr_kv_append", pages));
    if (!a) return cr_fail(ctx, CR_EINVAL, "cr_kv_append: args is NULL");
    if (!rotary) return cr_fail(ctx, CR_EINVAL, "cr_kv_append: rotary is NULL");
    if (layer >= pages->layers) return cr_fail(ctx, CR_EINVAL, "cr_kv_append: layer %u of %u", layer, pages->layers);
    if (a->n > (1u << 24) || a->n_tokens > (1u << 30) || a->q_heads > (1u << 20))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_append: too many entries, tokens or heads");
    if (a->reserved) return cr_fail(ctx, CR_EINVAL, "cr_kv_append: reserved must be 0");
    rope_in R;
    CR_TRY(rotary_check(ctx, "cr_kv_append", rotary, pages->head_dim, R));
    if (!a->n || !a->n_tokens) return CR_OK;
    if (!a->d_k || !a->d_v || !a->d_cu || (a->q_heads && (!a->d_q || !a->d_q_out)))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_append: NULL pointer");
    if (!aligned(a->d_k, a->k_token, a->k_head) || !aligned(a->d_v, a->v_token, a->v_head) ||
        !aligned(a->d_q, a->q_token, a->q_head) || !aligned(a->d_q_out, a->o_token, a->o_head))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_append: tensors must be 16-byte aligned, strides multiples of 8");
    if (a->q_heads && a->d_q == a->d_q_out && (a->q_token != a->o_token || a->q_head != a->o_head))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_append: in place, the queries' strides must be the same");
    return cr_append(ctx, "cr_kv_append", pages, layer, rotary, a);
}

extern "C" int cr_kv_read(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, const cr_read_args *a)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_kv_read");
    CR_TRY(cr_pages_check(ctx, "cr_kv_read", pages));
    if (!a) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: args is NULL");
    if (layer >= pages->layers) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: layer %u of %u", layer, pages->layers);
    const uint32_t n_tokens = a->n_tokens;
    if (a->n > (1u << 24) || n_tokens > (1u << 30)) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: too many entries or tokens");
    if (!n_tokens) return CR_OK;
    if (!a->d_k || !a->d_v || (a->n && !a->d_cu)) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: NULL pointer");
    if (!aligned(a->d_k, a->k_token, a->k_head) || !aligned(a->d_v, a->v_token, a->v_head))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_read: keys and values must be 16-byte aligned, strides multiples of 8");
    const pages_in P = cr_pages_input(ctx, pages);
    const read_in A = {static_cast<uint16_t *>(a->d_k), static_cast<uint16_t *>(a->d_v), a->k_token, a->k_head, a->v_token, a->v_head,
                       a->d_cu, a->d_seqs, a->d_start, a->n, n_tokens};
    const dim3 grid((n_tokens + kReadTokens - 1) / kReadTokens);
    if (!cr_in_8bit(pages->dtype)) return cr_launch_early(ctx, "k_kv_read", k_kv_read<true, false>, grid, kThreads, 0, P, A, layer);
    if (cr_is_bf16(pages->dtype)) return cr_launch_early(ctx, "k_kv_read", k_kv_read<true, true>, grid, kThreads, 0, P, A, layer);
    return cr_launch_early(ctx, "k_kv_read", k_kv_read<false, true>, grid, kThreads, 0, P, A, layer);
}
