// Rotary positions, writing of new tokens into pages (rotated, in 16 or 8 bits) and reading back
// (include/cacheroute.h).
//
// Angles.  The k-th pair's frequency is held as a 64-bit share of a full turn, so position times frequency is an integer
// product whose overflow drops whole turns: the angle of the furthest position is as exact as the nearest one's, where a
// 32-bit product would be off by 2^-24 of all the turns made.
//
// All three calls move each element once (2 bytes in, 2 or 1 out) and are bound by that, or by the latency of their
// dependent reads (list, length, table, page) where there are few tokens.  A lane holds four consecutive elements of a
// head; with the half layout its pairs' other elements are a quarter of the rotated part's lanes away (shuffles).
// Cosines and sines are made once for a CTA's tokens and shared by its heads.
#include <math.h>

#include "cr_attn_index.cuh"
#include "cr_pages.cuh"
#include "cr_tensor.cuh"

namespace {

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kSlice = 16;     // tokens whose cosines and sines a CTA holds
constexpr uint32_t kPairs = 64;     // of a head, at most
constexpr uint32_t kUnits = 4;      // heads that a warp holds at once
constexpr uint32_t kShortList = 1024;

struct rope_in {
    const uint64_t *turn;  // NULL: no rotation
    uint32_t pairs, layout;
    float scale, dir;      // dir: -1 inverse
};

struct rope_shared {
    float2 cs[kSlice * kPairs];  // [token][pair] (s cos, +-s sin)
};

// The slice's cosines and sines; pos(j): position of its j-th token.
template <typename POS>
__device__ __forceinline__ void make_angles(const rope_in &R, rope_shared &S, uint32_t count, POS pos)
{
    for (uint32_t i = threadIdx.x; i < count * R.pairs; i += kThreads) {
        const uint32_t j = i / R.pairs, k = i - j * R.pairs;
        const uint64_t turn = (uint64_t)(int64_t)pos(j) * R.turn[k];
        float sn, cs;
        sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn, &cs);  // half turns, -1 .. 1
        S.cs[j * kPairs + k] = make_float2(cs * R.scale, sn * R.scale * R.dir);
    }
}

// A lane's place in a token's head: elements d .. d+3 (sub: of which of the warp's tokens).
struct lane_place {
    uint32_t d, sub, per;  // per: tokens of a warp
    bool on, turns;
    int from;              // half layout: lane with the pairs' other elements
    bool second;           // half layout: these are the pairs' second elements
    __device__ __forceinline__ lane_place(uint32_t head_dim, const rope_in &R)
    {
        const uint32_t lane = threadIdx.x & 31, lanes = head_dim <= 64 ? 16 : 32, l = lane & (lanes - 1);
        per = 32 / lanes;
        sub = lane / lanes;
        d = 4 * l;
        on = d < head_dim;
        turns = R.turn && d < 2 * R.pairs;
        second = d >= R.pairs;
        from = (int)lane;
        if (turns && R.layout == CR_ROTARY_HALF) from = second ? (int)(lane - R.pairs / 4) : (int)(lane + R.pairs / 4);
    }
};
// What multiplies the lane's own elements and their partners.
struct lane_turn {
    float c[4], s[4];
    __device__ __forceinline__ void load(const rope_in &R, const rope_shared &S, const lane_place &L, uint32_t j)
    {
        if (!L.turns) return;
        if (R.layout == CR_ROTARY_HALF) {
            const float4 *p = reinterpret_cast<const float4 *>(S.cs + j * kPairs + (L.second ? L.d - R.pairs : L.d));
            const float4 a = p[0], b = p[1];
            c[0] = a.x, c[1] = a.z, c[2] = b.x, c[3] = b.z;
            s[0] = a.y, s[1] = a.w, s[2] = b.y, s[3] = b.w;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = L.second ? s[e] : -s[e];
        } else {
            const float4 a = *reinterpret_cast<const float4 *>(S.cs + j * kPairs + L.d / 2);
            c[0] = c[1] = a.x;
            c[2] = c[3] = a.z;
            s[0] = -a.y, s[1] = a.y;
            s[2] = -a.w, s[3] = a.w;
        }
    }
};

template <bool BF16>
__device__ __forceinline__ void unpack4(uint2 v, float *x)
{
    if (BF16) {
        x[0] = __uint_as_float(v.x << 16);
        x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16);
        x[3] = __uint_as_float(v.y & 0xffff0000u);
    } else {
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&v.x)),
                     b = __half22float2(*reinterpret_cast<const __half2 *>(&v.y));
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
    }
}
template <bool BF16>
__device__ __forceinline__ uint2 pack4(const float *x)
{
    return make_uint2(cr_pack16<BF16>(x[0], x[1]), cr_pack16<BF16>(x[2], x[3]));
}
// Four elements of the lane, rotated (the whole warp calls it).
template <bool BF16>
__device__ __forceinline__ void rotate4(const rope_in &R, const lane_place &L, const lane_turn &T, uint2 v, float *x)
{
    unpack4<BF16>(v, x);
    if (!R.turn) return;
    float y[4];
    if (R.layout == CR_ROTARY_HALF) {
        const uint2 o = make_uint2(__shfl_sync(~0u, v.x, L.from), __shfl_sync(~0u, v.y, L.from));
        unpack4<BF16>(o, y);
    } else {
        y[0] = x[1], y[1] = x[0], y[2] = x[3], y[3] = x[2];
    }
    if (L.turns) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(x[e], T.c[e], y[e] * T.s[e]);
    }
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
// four e4m3 numbers, the first lowest
__device__ __forceinline__ uint32_t pack_e4m3(const float *x)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ void unpack_e4m3(uint32_t v, float *x)
{
    uint32_t a, b;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((uint16_t)(v & 0xffff)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((uint16_t)(v >> 16)));
    const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&a)), q = __half22float2(*reinterpret_cast<const __half2 *>(&b));
    x[0] = p.x, x[1] = p.y, x[2] = q.x, x[3] = q.y;
}

// ---- rotating packed tokens ----------------------------------------------------------------------
struct rope_args {
    const uint16_t *x;
    uint16_t *o;
    uint64_t x_token, x_head, o_token, o_head;
    const int32_t *pos;
    uint32_t n_tokens, heads, head_dim;
};

// blockIdx.x: kSlice tokens; blockIdx.y: a share of the heads.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) k_rope(const __grid_constant__ rope_args A, const __grid_constant__ rope_in R)
{
    __shared__ __align__(16) rope_shared S;
    cr_launch_next();
    cr_wait_previous();
    const uint32_t t0 = blockIdx.x * kSlice, count = min(kSlice, A.n_tokens - t0);
    make_angles(R, S, count, [&](uint32_t j) { return A.pos[t0 + j]; });
    __syncthreads();
    const lane_place L(A.head_dim, R);
    const uint32_t h0 = (uint32_t)((uint64_t)A.heads * blockIdx.y / gridDim.y),
                   h1 = (uint32_t)((uint64_t)A.heads * (blockIdx.y + 1) / gridDim.y);
    const uint32_t groups = (h1 - h0 + kUnits - 1) / kUnits, tasks = (count + L.per - 1) / L.per * groups;
    for (uint32_t task = threadIdx.x >> 5; task < tasks; task += kWarps) {
        const uint32_t j = task / groups * L.per + L.sub, h = h0 + task % groups * kUnits;
        const bool on = L.on && j < count;
        const uint16_t *src = A.x + (uint64_t)(t0 + j) * A.x_token + L.d;
        uint2 v[kUnits];
#pragma unroll
        for (uint32_t u = 0; u < kUnits; ++u)
            v[u] = on && h + u < h1 ? *reinterpret_cast<const uint2 *>(src + (h + u) * A.x_head) : make_uint2(0, 0);
        lane_turn T;
        T.load(R, S, L, j < count ? j : 0);
        uint16_t *dst = A.o + (uint64_t)(t0 + j) * A.o_token + L.d;
#pragma unroll
        for (uint32_t u = 0; u < kUnits; ++u) {
            float x[4];
            rotate4<BF16>(R, L, T, v[u], x);
            const uint2 out = L.turns ? pack4<BF16>(x) : v[u];
            if (on && h + u < h1) *reinterpret_cast<uint2 *>(dst + (h + u) * A.o_head) = out;
        }
    }
}

// ---- writing into pages ----------------------------------------------------------------------------
struct append_in {
    const uint16_t *q, *k, *v;
    uint16_t *qo;
    uint64_t q_token, q_head, o_token, o_head, k_token, k_head, v_token, v_head;
    const int32_t *cu, *seqs;
    const int32_t *claim;  // long lists: the first entry of each row
    uint32_t n, n_tokens, q_heads, step_log2;  // step: positions of a slot
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
__global__ void __launch_bounds__(256) k_claim(int32_t *claim, const int32_t *seqs, uint32_t n, uint32_t n_seqs)
{
    cr_launch_next();
    cr_wait_previous();
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const int row = seqs[i];
        if (row >= 0 && (uint32_t)row < n_seqs) atomicMin(claim + row, (int)i);
    }
}

// What a CTA works on: up to `step` consecutive positions of a row, all in one block of a page.
struct slot_work {
    int t0, pos, count;     // first token, its position (the entry's first: 0, where there is no row), tokens
    int page;               // or -1: keys and values go nowhere
    uint32_t place;         // of the first token in its page
    bool lost;              // the positions are outside the row
};
// The slot of this CTA belongs to the last entry whose slots begin at or before it.  Every warp looks for itself.
__device__ __forceinline__ bool find_slot(const pages_in &P, const append_in &A, slot_work &W, uint32_t &entry)
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
    entry = lo;
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
    W.page = -1;
    W.place = (uint32_t)at.begin & (P.page - 1);
    W.lost = !have || at.begin < 0 || (uint64_t)at.begin >> P.page_log2 >= P.max_pages;
    if (!W.lost) {
        const int p = P.table[(uint64_t)row * P.max_pages + (uint32_t)(at.begin >> P.page_log2)];
        // pages that other rows name are not this row's to write (k_kv_write)
        if (p >= 0 && (uint32_t)p < P.n_pages && P.ref[p] <= 1) W.page = p;
        if (A.claim && A.claim[row] != (int)lo) W.page = -1;
    }
    return true;
}

template <bool BF16, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_kv_append(const __grid_constant__ pages_in P, const __grid_constant__ append_in A,
                                                        const __grid_constant__ rope_in R, uint32_t layer)
{
    __shared__ __align__(16) rope_shared S;
    extern __shared__ uint32_t dyn[];  // 8 bits: of each head's keys and values the largest magnitude, then the scales
    cr_launch_next();
    cr_wait_previous();
    slot_work W;
    uint32_t entry;
    if (!find_slot(P, A, W, entry)) return;
    if (A.seqs && !A.claim) {  // a row that an entry before this one names is that one's
        const int row = A.seqs[entry];
        bool twice = false;
        for (uint32_t i = threadIdx.x; i < entry; i += kThreads) twice |= A.seqs[i] == row;
        if (__syncthreads_or(twice)) W.page = -1;
    }
    const bool writes = W.page >= 0 && !W.lost;
    if (!writes && threadIdx.x == 0) atomicOr(P.status, CR_FLAG_BADPAGES);

    const uint32_t warp = threadIdx.x >> 5, y = blockIdx.y, ny = gridDim.y;
    const uint32_t q0 = (uint32_t)((uint64_t)A.q_heads * y / ny), q1 = (uint32_t)((uint64_t)A.q_heads * (y + 1) / ny);
    const uint32_t k0 = (uint32_t)((uint64_t)P.kv_heads * y / ny), nk = (uint32_t)((uint64_t)P.kv_heads * (y + 1) / ny) - k0;
    const lane_place L(P.head_dim, R);
    // units of a token: its key heads, then its value heads
    const uint32_t qg = (q1 - q0 + kUnits - 1) / kUnits, kg = writes ? (2 * nk + kUnits - 1) / kUnits : 0;
    uint32_t *top = dyn;
    float *scale = reinterpret_cast<float *>(dyn);
    uint8_t *kd = P.plane(2 * layer) + (W.page * P.page_stride << P.size_log2);
    uint8_t *vd = P.plane(2 * layer + 1) + (W.page * P.page_stride << P.size_log2);

    auto angles = [&](uint32_t s0, uint32_t n) {
        __syncthreads();
        if (R.turn) make_angles(R, S, n, [&](uint32_t j) { return W.pos + (int)(s0 + j); });
        __syncthreads();
    };
    // keys and values of a task: kUnits heads of L.per tokens
    auto load = [&](uint32_t t, bool in, uint32_t u0, uint2 *v) {
#pragma unroll
        for (uint32_t u = 0; u < kUnits; ++u) {
            const uint32_t i = u0 + u;
            v[u] = make_uint2(0, 0);
            if (in && i < 2 * nk)
                v[u] = i < nk ? *reinterpret_cast<const uint2 *>(A.k + (uint64_t)t * A.k_token + (k0 + i) * A.k_head + L.d)
                              : *reinterpret_cast<const uint2 *>(A.v + (uint64_t)t * A.v_token + (k0 + i - nk) * A.v_head + L.d);
        }
    };
    auto numbers = [&](const lane_turn &T, uint32_t i, uint2 v, float *x) {
        rotate4<BF16>(R, L, T, v, x);
        if (i >= nk) unpack4<BF16>(v, x);
    };

    if (E4M3) {
        for (uint32_t i = threadIdx.x; i < 2 * nk; i += kThreads) top[i] = 0;
    }
    float kept[kUnits][4];  // a task's numbers, where a warp has one only
    const bool once = (uint32_t)W.count <= kSlice && ((uint32_t)W.count + L.per - 1) / L.per * kg <= kWarps;
    // queries; keys' and values' largest magnitudes, or they themselves
    for (uint32_t s0 = 0; s0 < (uint32_t)W.count; s0 += kSlice) {
        const uint32_t n = min(kSlice, (uint32_t)W.count - s0), rounds = (n + L.per - 1) / L.per;
        angles(s0, n);
        for (uint32_t task = warp; task < rounds * (qg + kg); task += kWarps) {
            const bool is_q = task >= rounds * kg;
            const uint32_t i = is_q ? task - rounds * kg : task, per = is_q ? qg : kg;
            const uint32_t j = i / per * L.per + L.sub, u0 = i % per * kUnits;
            const bool in = L.on && j < n;
            const uint32_t t = (uint32_t)W.t0 + s0 + j;
            lane_turn T;
            uint2 v[kUnits];
            if (is_q) {
                const uint16_t *src = A.q + (uint64_t)t * A.q_token + L.d;
                const uint32_t h = q0 + u0;
#pragma unroll
                for (uint32_t u = 0; u < kUnits; ++u)
                    v[u] = in && h + u < q1 ? *reinterpret_cast<const uint2 *>(src + (h + u) * A.q_head) : make_uint2(0, 0);
                T.load(R, S, L, j < n ? j : 0);
                uint16_t *dst = A.qo + (uint64_t)t * A.o_token + L.d;
#pragma unroll
                for (uint32_t u = 0; u < kUnits; ++u) {
                    float x[4];
                    rotate4<BF16>(R, L, T, v[u], x);
                    uint2 out = L.turns ? pack4<BF16>(x) : v[u];
                    if (W.lost) out = make_uint2(0, 0);
                    if (in && h + u < q1) *reinterpret_cast<uint2 *>(dst + (h + u) * A.o_head) = out;
                }
                continue;
            }
            load(t, in, u0, v);
            T.load(R, S, L, j < n ? j : 0);
            const uint64_t at = (uint64_t)(W.place + s0 + j) * P.token_stride + L.d;
#pragma unroll
            for (uint32_t u = 0; u < kUnits; ++u) {
                float x[4];
                numbers(T, u0 + u, v[u], x);
                if (E4M3) {
                    float m = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = fabsf(x[e]);
                        m = a < e4m3_range<BF16>::kInf ? fmaxf(m, a) : m;
                        kept[u][e] = x[e];
                    }
                    const uint32_t all = __reduce_max_sync(~0u, __float_as_uint(m));
                    if ((threadIdx.x & 31) == 0 && u0 + u < 2 * nk) atomicMax(top + u0 + u, all);
                } else if (in && u0 + u < 2 * nk) {
                    const bool key = u0 + u < nk;
                    const uint64_t to = at + (k0 + u0 + u - (key ? 0 : nk)) * P.head_stride;
                    *reinterpret_cast<uint2 *>((key ? kd : vd) + 2 * to) = key && L.turns ? pack4<BF16>(x) : v[u];
                }
            }
        }
    }
    if (!E4M3 || !writes) return;

    // the blocks' powers
    __syncthreads();
    const uint32_t nb_log2 = P.page_log2 - P.block_log2, block = W.place >> P.block_log2, before = W.place & ((1u << P.block_log2) - 1);
    for (uint32_t i = threadIdx.x; i < 2 * nk; i += kThreads) {
        const uint32_t h = k0 + (i < nk ? i : i - nk);
        float *at = P.scales(2 * layer + (i >= nk), (uint32_t)W.page) + (h << nb_log2) + block;
        float now = block_power<BF16>(__uint_as_float(top[i]));
        float ratio = 1.f;
        if (before) {
            const float old = *at;
            now = fmaxf(now, old);
            ratio = old / now;
        }
        *at = now;
        scale[i] = now;
        scale[2 * nk + i] = ratio;
    }
    __syncthreads();
    // the tokens that were there, where the power has grown
    for (uint32_t i = before ? warp : 2 * nk; i < 2 * nk; i += kWarps) {
        const float ratio = scale[2 * nk + i];
        if (ratio == 1.f) continue;
        const uint32_t h = k0 + (i < nk ? i : i - nk);
        uint8_t *base = (i < nk ? kd : vd) + h * P.head_stride + L.d;
        for (uint32_t j = L.sub; j < before; j += L.per) {
            uint32_t *at = reinterpret_cast<uint32_t *>(base + (uint64_t)(W.place - before + j) * P.token_stride);
            if (!L.on) continue;
            float x[4];
            unpack_e4m3(*at, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= ratio;
            *at = pack_e4m3(x);
        }
    }
    for (uint32_t s0 = 0; s0 < (uint32_t)W.count; s0 += kSlice) {
        const uint32_t n = min(kSlice, (uint32_t)W.count - s0), rounds = (n + L.per - 1) / L.per;
        if ((uint32_t)W.count > kSlice) angles(s0, n);
        for (uint32_t task = warp; task < rounds * kg; task += kWarps) {
            const uint32_t j = task / kg * L.per + L.sub, u0 = task % kg * kUnits;
            const bool in = L.on && j < n;
            if (!once) {
                uint2 v[kUnits];
                lane_turn T;
                load((uint32_t)W.t0 + s0 + j, in, u0, v);
                T.load(R, S, L, j < n ? j : 0);
#pragma unroll
                for (uint32_t u = 0; u < kUnits; ++u) numbers(T, u0 + u, v[u], kept[u]);
            }
            const uint64_t at = (uint64_t)(W.place + s0 + j) * P.token_stride + L.d;
#pragma unroll
            for (uint32_t u = 0; u < kUnits; ++u) {
                const uint32_t i = u0 + u;
                if (!in || i >= 2 * nk) continue;
                const float by = 1.f / scale[i], most = scale[i] >= ldexpf(1.f, e4m3_range<BF16>::kMax) ? 240.f : 448.f;
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = kept[u][e];
                    x[e] = fabsf(a) < e4m3_range<BF16>::kInf ? fminf(fmaxf(a * by, -most), most) : __int_as_float(0x7fffffff);
                }
                const uint64_t to = at + (k0 + (i < nk ? i : i - nk)) * P.head_stride;
                *reinterpret_cast<uint32_t *>((i < nk ? kd : vd) + to) = pack_e4m3(x);
            }
        }
    }
}

// ---- reading back ----------------------------------------------------------------------------------
struct read_in {
    uint16_t *k, *v;
    uint64_t k_token, k_head, v_token, v_head;
    const int32_t *cu, *seqs, *start;
    uint32_t n, n_tokens;
};

// A warp per token; a lane takes 8 elements at a time.
template <bool BF16, bool E4M3>
__global__ void __launch_bounds__(128) k_kv_read(const __grid_constant__ pages_in P, const __grid_constant__ read_in A, uint32_t layer)
{
    cr_launch_next();
    cr_wait_previous();
    const uint64_t t = ((uint64_t)blockIdx.x * 128 + threadIdx.x) >> 5;
    if (t >= A.n_tokens) return;
    const uint32_t lane = threadIdx.x & 31;
    uint32_t lo = 0, span = A.n + 1;
    while (span > 1) {
        const uint32_t step = (span + 31) / 32, i = lo + lane * step;
        const bool in = lane * step < span && A.cu[i] <= (int)t;
        const uint32_t some = __ballot_sync(~0u, in), last = some ? 31 - __clz(some) : 0;
        lo += last * step;
        span = min(step, span - last * step);
    }
    bool ok = lo < A.n && A.cu[lo] <= (int)t && (int)t < A.cu[lo + 1];
    uint32_t page = 0, place = 0;
    if (ok) {
        const int row = A.seqs ? A.seqs[lo] : (int)lo;
        ok = row >= 0 && (uint32_t)row < P.n_seqs;
        if (ok) {
            const int len = P.lens[row];
            const long long pos = (A.start ? (long long)A.start[lo] : (long long)len - ((long long)A.cu[lo + 1] - A.cu[lo])) + ((int)t - A.cu[lo]);
            ok = pos >= 0 && pos < len && ((uint64_t)pos >> P.page_log2) < P.max_pages;
            if (ok) {
                const int p = P.table[(uint64_t)row * P.max_pages + (uint32_t)(pos >> P.page_log2)];
                ok = p >= 0 && (uint32_t)p < P.n_pages;
                page = (uint32_t)p;
                place = (uint32_t)pos & (P.page - 1);
            }
        }
    }
    if (!ok && lane == 0) atomicOr(P.status, CR_FLAG_BADPAGES);
    const uint32_t per = P.head_dim / 8, words = P.kv_heads * per;
    const uint64_t at = page * P.page_stride + place * P.token_stride;
    const uint32_t nb_log2 = P.page_log2 - P.block_log2;
    for (uint32_t i = lane; i < words; i += 32) {
        const uint32_t h = i / per, d = (i - h * per) * 8;
#pragma unroll
        for (uint32_t c = 0; c < 2; ++c) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (ok) {
                const uint8_t *src = P.plane(2 * layer + c) + ((at + h * P.head_stride + d) << P.size_log2);
                if (E4M3) {
                    const uint2 q = *reinterpret_cast<const uint2 *>(src);
                    const float f = P.scales(2 * layer + c, page)[(h << nb_log2) + (place >> P.block_log2)];
                    float x[8];
                    unpack_e4m3(q.x, x);
                    unpack_e4m3(q.y, x + 4);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= f;
                    v = make_uint4(cr_pack16<BF16>(x[0], x[1]), cr_pack16<BF16>(x[2], x[3]), cr_pack16<BF16>(x[4], x[5]),
                                   cr_pack16<BF16>(x[6], x[7]));
                } else {
                    v = *reinterpret_cast<const uint4 *>(src);
                }
            }
            uint16_t *dst = c ? A.v + t * A.v_token + h * A.v_head + d : A.k + t * A.k_token + h * A.k_head + d;
            *reinterpret_cast<uint4 *>(dst) = v;
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

bool aligned(const void *p, uint64_t a, uint64_t b) { return ((uintptr_t)p & 15) == 0 && (a & 7) == 0 && (b & 7) == 0; }

}  // namespace

extern "C" int cr_rope(cr_ctx *ctx, const cr_rotary *rotary, uint32_t dtype, const void *d_x, uint64_t x_token, uint64_t x_head,
                       void *d_out, uint64_t o_token, uint64_t o_head, uint32_t n_tokens, uint32_t heads, uint32_t head_dim,
                       const int32_t *d_pos)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_rope");
    if (!rotary) return cr_fail(ctx, CR_EINVAL, "cr_rope: rotary is NULL");
    if (dtype > CR_DTYPE_FP16) return cr_fail(ctx, CR_EINVAL, "cr_rope: dtype %u", dtype);
    if (!head_dim || head_dim > 128 || (head_dim & 7)) return cr_fail(ctx, CR_EINVAL, "cr_rope: head_dim %u: a multiple of 8, 8..128", head_dim);
    rope_in R;
    CR_TRY(rotary_check(ctx, "cr_rope", rotary, head_dim, R));
    if (n_tokens > (1u << 30) || heads > (1u << 20)) return cr_fail(ctx, CR_EINVAL, "cr_rope: too many tokens or heads");
    if (!n_tokens || !heads) return CR_OK;
    if (!d_x || !d_out || !d_pos) return cr_fail(ctx, CR_EINVAL, "cr_rope: NULL pointer");
    if (!aligned(d_x, x_token, x_head) || !aligned(d_out, o_token, o_head))
        return cr_fail(ctx, CR_EINVAL, "cr_rope: tensors must be 16-byte aligned, strides multiples of 8");
    if (d_x == d_out && (x_token != o_token || x_head != o_head))
        return cr_fail(ctx, CR_EINVAL, "cr_rope: in place, the strides must be the same");
    const rope_args A = {static_cast<const uint16_t *>(d_x), static_cast<uint16_t *>(d_out), x_token, x_head, o_token, o_head,
                         d_pos, n_tokens, heads, head_dim};
    const uint32_t blocks = (n_tokens + kSlice - 1) / kSlice;
    // few tokens: several CTAs share a slice's heads
    const uint32_t split = max(1u, min((heads + kUnits - 1) / kUnits, 4 * (uint32_t)ctx->num_sms / blocks));
    if (dtype == CR_DTYPE_BF16) return cr_launch_early(ctx, "k_rope", k_rope<true>, dim3(blocks, split), kThreads, 0, A, R);
    return cr_launch_early(ctx, "k_rope", k_rope<false>, dim3(blocks, split), kThreads, 0, A, R);
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
        CR_TRY(cr_launch_early(ctx, "k_claim", k_claim, dim3(blocks), 256, 0, claim, A.seqs, A.n, P.n_seqs));
        A.claim = claim;
    }
    const uint64_t slots = ((uint64_t)A.n_tokens >> A.step_log2) + 2ull * A.n;
    const uint64_t want = 8ull * (uint32_t)ctx->num_sms / slots;
    uint32_t split = want < 1 ? 1 : (want < pg->kv_heads ? (uint32_t)want : pg->kv_heads);
    const size_t smem = e4m3 ? 16 * (size_t)((pg->kv_heads + split - 1) / split) : 0;
    // more than 1,024 heads would need more than the default shared memory
    if (smem > 16 * 1024) split = (pg->kv_heads + 1023) / 1024;
    const dim3 grid((uint32_t)slots, split);
    const size_t bytes = e4m3 ? 16 * (size_t)((pg->kv_heads + split - 1) / split) : 0;
    if (cr_is_bf16(pg->dtype))
        return e4m3 ? cr_launch_early(ctx, "k_kv_append", k_kv_append<true, true>, grid, kThreads, bytes, P, A, R, layer)
                    : cr_launch_early(ctx, "k_kv_append", k_kv_append<true, false>, grid, kThreads, bytes, P, A, R, layer);
    return e4m3 ? cr_launch_early(ctx, "k_kv_append", k_kv_append<false, true>, grid, kThreads, bytes, P, A, R, layer)
                : cr_launch_early(ctx, "k_kv_append", k_kv_append<false, false>, grid, kThreads, bytes, P, A, R, layer);
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

extern "C" int cr_kv_read(cr_ctx *ctx, const cr_kv_pages *pages, uint32_t layer, void *d_k, uint64_t k_token, uint64_t k_head,
                          void *d_v, uint64_t v_token, uint64_t v_head, const int32_t *d_cu, const int32_t *d_seqs,
                          const int32_t *d_start, uint32_t n, uint32_t n_tokens)
{
    if (!ctx) return CR_EINVAL;
    cr_nvtx_range range("cr_kv_read");
    CR_TRY(cr_pages_check(ctx, "cr_kv_read", pages));
    if (layer >= pages->layers) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: layer %u of %u", layer, pages->layers);
    if (n > (1u << 24) || n_tokens > (1u << 30)) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: too many entries or tokens");
    if (!n || !n_tokens) return CR_OK;
    if (!d_k || !d_v || !d_cu) return cr_fail(ctx, CR_EINVAL, "cr_kv_read: NULL pointer");
    if (!aligned(d_k, k_token, k_head) || !aligned(d_v, v_token, v_head))
        return cr_fail(ctx, CR_EINVAL, "cr_kv_read: keys and values must be 16-byte aligned, strides multiples of 8");
    const pages_in P = cr_pages_input(ctx, pages);
    const read_in A = {static_cast<uint16_t *>(d_k), static_cast<uint16_t *>(d_v), k_token, k_head, v_token, v_head, d_cu, d_seqs,
                       d_start, n, n_tokens};
    const dim3 grid((n_tokens + 3) / 4);
    if (!cr_in_8bit(pages->dtype)) return cr_launch_early(ctx, "k_kv_read", k_kv_read<true, false>, grid, 128, 0, P, A, layer);
    if (cr_is_bf16(pages->dtype)) return cr_launch_early(ctx, "k_kv_read", k_kv_read<true, true>, grid, 128, 0, P, A, layer);
    return cr_launch_early(ctx, "k_kv_read", k_kv_read<false, true>, grid, 128, 0, P, A, layer);
}
