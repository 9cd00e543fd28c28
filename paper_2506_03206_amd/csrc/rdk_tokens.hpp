// Tokens of a row held against the row while it is read once: the sums that its log probabilities and its entropy are formed of, and the tokens' ranks.
//
// With M the row's largest value, Z' the sum over all other entries of exp((x - M) / T) (weights: of x / M) and U the sum of exp((x - M) / T) (x - M) / T:
//   log s_j = (x_j - M) / T - log(1 + Z'),    entropy = log(1 + Z') - U / (1 + Z'),
// every term of which has one sign: a row that is sure of its best entry has an entropy and a log probability of that entry far below
// the rounding of a sum that begins with 1, and they keep their own 24 bits this way.
#pragma once
#include <algorithm>
#include <cmath>

#include "rdk_select.hpp"
#include "rdk_vec.hpp"

namespace rdk {

constexpr int kMaxTokens = 16;        // given tokens of a row: a lane each
constexpr int kTokenRoundVecs = 4;    // 16-byte vectors of a thread in a round
constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;

// (x - M) / T by way of (x - M) unit, with a power of two that makes it a number of about its final size: nothing overflows that the result does not, at whatever T,
// and the bits are those of x - M.
struct Distance {
    float unit;   // 1 / T to a power of two; 1/2 at temperatures below 2
    float inv;    // to units of log e
    float c;      // to units of log 2

    static Distance over(float T)
    {
        const float unit = std::ldexp(1.f, -std::min(std::max(std::ilogb(T), 1), 126));
        const float inv = T < 2.f ? 1.f / T * 2.f : 1.f / (T * unit);
        return Distance{unit, inv, inv * kLog2e};
    }
    // Of sums of exponentials times distances: at temperatures below 2^-10, too, a number of about the size over T, so that products with exponentials that are next to
    // nothing keep their bits.  (Above, half of x - M is near enough, and finite for any two numbers: masks of the lowest value cost nothing.)
    static Distance in_sums(float T)
    {
        const int e = std::ilogb(T) + 1;
        if (e > -10) return over(T);
        const float unit = std::ldexp(1.f, -e), inv = 1.f / (T * unit);
        return Distance{unit, inv, inv * kLog2e};
    }
    __device__ __forceinline__ float of(float x, float m) const { return fmaf(x, unit, -m * unit); }
};

// What a part of a row, or a row, comes to.  m: the largest value; rest: the others' sum relative to it (the largest itself counts 1 beside it);
// pull: the sum of their terms times their distance to it, in units of log e (<= 0).  Of a part without unmasked entries m is none.
struct RowSum {
    float m, rest, pull;
};

struct TokenArgs {
    const int32_t *slot_of;   // target id -> slot, or NULL: ids are places in the row
    const int32_t *kept_ids;  // slot -> target id, with slot_of
    int ids;                  // ids below this are known there
    int C;
    Distance from_most;
    Distance in_sums;         // those in the sums of rows in registers
    float far;                // a largest value whose product with its unit may be no number
    float c, margin;          // c = log2(e) / T; margin: what references are exceeded by before they are replaced, 8 / c
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *rank;
    float4 *stats;            // m, rest, pull / (1 + rest), unused
    float4 *part_sum;         // [B, parts], at most 64 parts: a lane each
    int32_t *part_rank;       // [B, C, parts]
};

constexpr int kNoToken = -2, kUnknown = -1;   // a place that is none: nothing was asked, or an id that the vocabulary does not hold

template <int KIND>
__device__ __forceinline__ float no_value() { return KIND == RDK_PROB_F32 ? 0.f : -INFINITY; }

// The place of a token in the row.
__device__ __forceinline__ int place_of(int id, const int32_t *slot_of, int ids)
{
    if (id < 0) return kNoToken;
    if (id >= ids) return kUnknown;
    return slot_of ? max(slot_of[id], kUnknown) : id;
}

// A power of two by which weights up to m come to lie below 4, and its logarithm.  (Weights below 2^-126 stay below 1.)
__device__ __forceinline__ int weight_exponent(float m) { return min(max((int)(__float_as_uint(m) >> 23) & 0xFF, 1) - 127, 126); }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }

constexpr float kWide = 0x1p22f;

// The sums that a lane, and later a workgroup, holds.  With y = x log2(e) / T (weights: log2 x) and a whole number ref that the largest y exceeds by about 8.5 at most (terms up to 2^8.5):
//   sum = sum 2^(y - ref),   pull = sum 2^(y - ref) (y - ref)
// A whole reference is exact in a product and sum of one rounding, so an entry costs an addition less than with a difference first, and a change of it is
// a power of two.  (Rows with y beyond +-2^22, where a product is rounded by more than a fraction, are read again: kWide.)
template <int KIND>
struct Sums {
    float m, sum, pull;
    float ref, high;
    float scale;   // of weights, 2^-ref

    __device__ __forceinline__ void clear()
    {
        m = high = no_value<KIND>();
        sum = pull = ref = 0.f;
        scale = 1.f;
    }

    // of a largest value
    static __device__ __forceinline__ float reference(float x, float c)
    {
        return KIND == RDK_PROB_F32 ? (float)weight_exponent(x) : __builtin_rintf(fminf(fmaxf(weight_reference(x) * c, -kWide), kWide));
    }

    // to another reference
    __device__ __forceinline__ void move(float to)
    {
        const float by = ref - to, f = __builtin_amdgcn_exp2f(by);
        pull = sum == 0.f || f == 0.f ? 0.f : f * fmaf(by, sum, pull);
        sum = sum == 0.f ? 0.f : f * sum;
        ref = to;
    }

    __device__ __forceinline__ void raise(float x, float c, float margin)
    {
        const float to = reference(x, c);
        move(to);
        if constexpr (KIND == RDK_PROB_F32) {
            scale = power_of_two(-(int)to);
            high = power_of_two((int)to + 8);
        } else {
            high = x + margin;
        }
    }

    // the terms of a vector, its own sums first: long rows are sums of sums
    template <int E>
    __device__ __forceinline__ void add(const float (&x)[E], float c)
    {
        float s = 0.f, p = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            float e, d;
            if constexpr (KIND == RDK_PROB_F32) {
                e = x[i] * scale;
                d = __builtin_amdgcn_logf(fmaxf(e, 0x1p-126f));   // (log2)
            } else {
                d = fmaf(x[i], c, -ref);
                e = __builtin_amdgcn_exp2f(d);
            }
            s = i == 0 ? e : s + e;
            p = i == 0 ? e * d : fmaf(e, d, p);
        }
        if (KIND != RDK_PROB_F32 && p != p) {   // 0 times the distance of a masked entry: such distances are held finite.  (NaN is in the sum.)
            p = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float d = fmaf(x[i], c, -ref);
                p = fmaf(__builtin_amdgcn_exp2f(d), fmaxf(d, -0x1p126f), p);
            }
        }
        sum += s;
        pull += p;
    }
};

template <int THREADS>
struct TokenShared {
    static constexpr int kWaves = THREADS / kWave;
    struct {
        float m, sum, pull;            // of a wavefront, relative to what its own largest value asks for
        float sum_besides, pull_besides;   // of all lanes but the first that has the largest value
        int holder;
    } wave[kWaves];
    float others[kWaves], other_pull[kWaves];
    int ties[kWaves];
    int rank[kWaves][kMaxTokens];
};

// Entries before a token of a thread's own vectors, [token][thread]: a word that only this thread reads and writes.  Of as many tokens as there are, so that
// workgroups of few tokens lie beside each other (16 always: four fused passes a unit become three, 1024 rows of 151936 bf16 logits 72 -> 77 us).
template <int THREADS>
__device__ __forceinline__ uint32_t &before_token(int c)
{
    extern __shared__ uint32_t before[];
    return before[c * THREADS + (int)threadIdx.x];
}
inline uint32_t before_tokens_bytes(const TokenArgs &a, int threads) { return a.rank ? (uint32_t)(a.C * threads * 4) : 0; }

// log probability of an entry x of a row with the largest value m, log_all = log(1 + rest)
template <int KIND>
__device__ __forceinline__ float log_share(float x, float m, float log_all, const Distance &by)
{
    if (KIND == RDK_PROB_F32) {
        if (!(x > 0.f)) return x == 0.f ? -INFINITY : x;
        // (the ratio of weights that far apart may be no normal number, which has fewer bits)
        return (x < m * 0x1p-100f ? logf(x * 0x1p64f) - (logf(m) + 64.f * kLn2) : logf(x / m)) - log_all;
    }
    return x == -INFINITY ? -INFINITY : by.of(x, m) * by.inv - log_all;
}

// The outputs of a row, by one wavefront; count: of lane c, entries before token c.
template <int KIND>
__device__ __forceinline__ void write_tokens(const TokenArgs &a, int64_t row, RowSum s, int place, float value, int count)
{
    const bool none = s.m == no_value<KIND>() && s.rest == 0.f;
    const float log_all = log1pf(s.rest);
    if (lane_id() < a.C) {
        const int64_t o = row * a.C + lane_id();
        float lp = place == kNoToken ? 0.f : -INFINITY;
        if (place >= 0 && !none) lp = log_share<KIND>(value, s.m, log_all, a.from_most);
        a.logprob[o] = lp;
        if (a.rank) a.rank[o] = place >= 0 && lp > -INFINITY ? count : -1;
    }
    if (lane_id() == 0) {
        const float pull = s.pull / (1.f + s.rest);
        if (a.entropy) a.entropy[row] = none ? 0.f : log_all - pull;
        if (a.stats) a.stats[row] = make_float4(s.m, s.rest, pull, 0.f);
    }
}

// sum over the 64 lanes of a whole number, in every lane
__device__ __forceinline__ int wave_count(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// (by value: a cast of an element of a vector takes the vector's first)
__device__ __forceinline__ s16x2 s16x2_of(uint32_t w) { return __builtin_bit_cast(s16x2, w); }
__device__ __forceinline__ u16x2 u16x2_of(uint32_t w) { return __builtin_bit_cast(u16x2, w); }

// Entries of a thread's vectors before a token of the value v that lies in the vector `first`; they begin with `base` and stand THREADS apart.  In vectors before a
// token's own the entries that equal it count too.  Nothing waits for the mask of a comparison: pairs of bf16 values are taken as signed whole numbers, of which those
// below 0 have their order turned round with all others (`turn`), and counted in 16 bits each; of fp32 values the signs of differences are gathered.  Bounds are a
// wavefront's but where the token lies among the vectors.
template <int KIND, int THREADS, int VECS>
__device__ __forceinline__ uint32_t entries_before(u32x4 (&now)[VECS], int base, int first, float v)
{
    typedef Vec<KIND> V;
#pragma unroll
    for (int j = 0; j < VECS; ++j) V::again(now[j]);   // (or what is made of them for every token alike would be kept beside them)
    const bool all_before = first >= base + VECS * THREADS, none_before = first <= base;
    uint32_t n = 0;
    if constexpr (KIND == RDK_LOGIT_BF16) {
        // above v: turned if v < 0;  at least v: turned if v <= 0, as -0 is the next below 0 in that order and equals it
        const uint32_t half = __float_as_uint(v + 0.f) >> 16;
        const uint32_t turn_above = v < 0.f ? 0x7FFF7FFFu : 0u, turn_least = v <= 0.f ? 0x7FFF7FFFu : 0u;
        const uint32_t above = (half ^ (turn_above & 0xFFFFu)) * 0x10001u;
        const uint32_t least = (v == 0.f ? 0xFFFEu : ((half ^ (turn_least & 0xFFFFu)) - 1u) & 0xFFFFu) * 0x10001u;
        s16x2 counts = {0, 0};
        auto take = [&](u32x4 x, uint32_t bound, uint32_t turn) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) counts -= __builtin_elementwise_sub_sat(s16x2_of(bound), s16x2_of(x[i] ^ turn)) >> 15;
        };
        if (all_before || none_before) {
            const uint32_t bound = all_before ? least : above, turn = all_before ? turn_least : turn_above;
#pragma unroll
            for (int j = 0; j < VECS; ++j) take(now[j], bound, turn);
        } else {
#pragma unroll
            for (int j = 0; j < VECS; ++j) {
                const bool before = base + j * THREADS + (int)threadIdx.x < first;
                take(now[j], before ? least : above, before ? turn_least : turn_above);
            }
        }
        n = __builtin_bit_cast(uint32_t, counts);
        n = (n & 0xFFFFu) + (n >> 16);
    } else {
        // above v: v - x < 0;  at least v: not x - v < 0.  (No bound beside v, which below the lowest finite value would be -inf, and -inf - -inf no number.)
        static_assert(V::kLen * VECS <= 32, "a bit each");
        const float above = v + 0.f, least = 0.f - v;   // (0 - 0 has no sign, -0 - 0 has)
        auto take = [&](u32x4 x, float factor, float bound, uint32_t turn) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) n = __builtin_amdgcn_alignbit(n, __float_as_uint(fmaf(__uint_as_float(x[i]), factor, bound)), 31);
            n ^= turn;
        };
        if (all_before || none_before) {
            const float factor = all_before ? 1.f : -1.f, bound = all_before ? least : above;
            const uint32_t turn = all_before ? 15u : 0u;
#pragma unroll
            for (int j = 0; j < VECS; ++j) take(now[j], factor, bound, turn);
        } else {
#pragma unroll
            for (int j = 0; j < VECS; ++j) {
                const bool before = base + j * THREADS + (int)threadIdx.x < first;
                take(now[j], before ? 1.f : -1.f, before ? least : above, before ? 15u : 0u);
            }
        }
        n = __popc(n);
    }
    return n;
}

// A part of a row read by a workgroup in rounds of four vectors a thread.  A lane's sums are relative to a value that it has seen; the lane that ends
// with the largest of all has that entry's 1 in its sum, in whose rounding its other entries may be lost: where that matters (all others
// together come to less than it) this lane's vectors are read again, out of the cache, a vector to a thread, and summed without it.  Entries before a token in the
// order of rdk_topk are those above its value, and those that equal it at a lower place: in vectors before its own the bound is the next number below.
template <int KIND, int THREADS, bool RANKS>
struct TokenPass {
    typedef Vec<KIND> V;
    typedef TokenShared<THREADS> Shared;
    static constexpr int kWaves = THREADS / kWave;
    Sums<KIND> s;
    int place, here, count;   // of lane c, token c in every wavefront: its place in the row and from the part's beginning, entries before it
    float value;

    // The part's entries are first .. last - 1 of a row that ends at `end`.
    __device__ __forceinline__ void begin(const TokenArgs &a, int64_t row, const void *xr, int first, int last, int end)
    {
        s.clear();
        place = kNoToken;
        here = count = 0;
        value = NAN;   // (nothing is before none)
        if (RANKS && a.rank)
            for (int c = 0; c < a.C; ++c) before_token<THREADS>(c) = 0;
        if (lane_id() < a.C) place = place_of(a.tokens[row * a.C + lane_id()], a.slot_of, a.ids);
        if (place >= 0) {
            here = place - first;
            // its vector of the row (parts begin with whole vectors), and in it the entries before it that equal it, which the bounds of vectors pass over
            const int own = place & ~(V::kLen - 1);
            float v[V::kLen];
            V::to(V::load(xr, own, end), v);
            value = v[0];
#pragma unroll
            for (int e = 1; e < V::kLen; ++e) value = place - own == e ? v[e] : value;
            if (RANKS && threadIdx.x < kWave && here >= 0 && own + V::kLen <= last)
#pragma unroll
                for (int e = 0; e < V::kLen - 1; ++e) count += (own + e < place) & (v[e] == value);
        }
    }

    // One value of a lane (none where it has none), at the place `at` of the row.
    __device__ __forceinline__ void single(const TokenArgs &a, float x, int at)
    {
        s.m = fmaxf(s.m, x);
        if (x > s.high) s.raise(x, a.c, a.margin);
        s.add({x}, a.c);
        if (RANKS)
            for (int c = 0; c < a.C; ++c) {
                const int to = lane_value(place, c);
                const float v = lane_value(value, c);
                const int before = __popcll(__ballot(x > v || (x == v && at < to)));
                if (lane_id() == c) count += before;
            }
    }

    // A lane's vector; returns its largest value.
    __device__ __forceinline__ float vector(const TokenArgs &a, u32x4 &raw)
    {
        float v[V::kLen];
        V::to(raw, v);
        const float most = V::largest(v, no_value<KIND>());
        if (most > s.high) s.raise(most, a.c, a.margin);
        s.add(v, a.c);
        V::again(raw);
        return most;
    }

    // Entries of a round before the tokens; its vectors begin with `base` of the part, most is the lane's largest value of the round.  A thread's counts are
    // its own until the end.
    __device__ __forceinline__ void ranks(const TokenArgs &a, u32x4 (&now)[kTokenRoundVecs], float most, int base)
    {
#pragma unroll 1
        for (int c = 0; c < a.C; ++c) {
            const float v = lane_value(value, c);
            if (__ballot(most >= v) == 0) continue;
            const int first = lane_value(here, c) >> (V::kLen == 8 ? 3 : 2);   // (-1 or less: it lies before the part)
            __hip_atomic_fetch_add(&before_token<THREADS>(c), entries_before<KIND, THREADS>(now, base, first, v), __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_WAVEFRONT);
        }
    }

    // The part's sums in every thread; from: where the part begins, with `whole` vectors and `behind` values after them, one of the first threads each.
    __device__ __forceinline__ RowSum finish(const TokenArgs &a, const char *from, int whole, int behind, Shared &sh)
    {
        const int tid = threadIdx.x, wid = tid / kWave;
        // every wavefront relative to its own largest value first, then all relative to the part's: one meeting
        const float wave_most = wave_max(s.m);
        if (s.sum != 0.f) s.move(s.reference(wave_most, a.c));
        const uint64_t who = __ballot(s.m == wave_most);
        const bool first = who && lane_id() == __ffsll((unsigned long long)who) - 1;
        const float sum_w = wave_sum(s.sum), pull_w = wave_sum(s.pull), sum_b = wave_sum(first ? 0.f : s.sum), pull_b = wave_sum(first ? 0.f : s.pull);
        if (first) sh.wave[wid].holder = tid;
        if (lane_id() == 0) {
            sh.wave[wid].m = wave_most;
            sh.wave[wid].sum = sum_w;
            sh.wave[wid].pull = pull_w;
            sh.wave[wid].sum_besides = sum_b;
            sh.wave[wid].pull_besides = pull_b;
        }
        if (RANKS) {
            for (int c = 0; a.rank && c < a.C; c += 4) {   // four at a time on their way
                int own[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) own[i] = (int)before_token<THREADS>(min(c + i, a.C - 1));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int all = wave_count(own[i]);
                    if (lane_id() == c + i) count += all;
                }
            }
            if (lane_id() < a.C) sh.rank[wid][lane_id()] = count;
        }
        __syncthreads();
        float m = sh.wave[0].m;
        int holds = 0;   // the first wavefront that has the largest value
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            if (sh.wave[w].m > m) holds = w;
            m = fmaxf(m, sh.wave[w].m);
        }
        const float ref = s.reference(m, a.c), scale = KIND == RDK_PROB_F32 ? power_of_two(-(int)ref) : 1.f;
        float sum = 0.f, pull = 0.f, others = 0.f, other_pull = 0.f;
        auto add = [&](float &to, float &to_pull, float wave_m, float x, float p) __attribute__((always_inline)) {
            if (x == 0.f) return;
            Sums<KIND> t;
            t.sum = x;
            t.pull = p;
            t.ref = s.reference(wave_m, a.c);
            t.move(ref);
            to += t.sum;
            to_pull += t.pull;
        };
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            add(sum, pull, sh.wave[w].m, sh.wave[w].sum, sh.wave[w].pull);
            if (w == holds) add(others, other_pull, sh.wave[w].m, sh.wave[w].sum_besides, sh.wave[w].pull_besides);
            else add(others, other_pull, sh.wave[w].m, sh.wave[w].sum, sh.wave[w].pull);
        }
        const bool some = m > no_value<KIND>() && m < INFINITY;
        if (!some) return RowSum{m, m > 0.f ? NAN : sum - sum, 0.f};   // (NaN where there is one or an infinity, 0 where all is masked)
        // what the largest entry counts, and its distance from the reference
        const float log_own = KIND == RDK_PROB_F32 ? __builtin_amdgcn_logf(m * scale) : fmaf(m, a.c, -ref);
        const float own = KIND == RDK_PROB_F32 ? m * scale : __builtin_amdgcn_exp2f(log_own), inv = 1.f / own;
        const bool wide = KIND != RDK_PROB_F32 && !(fabsf(m * a.c) < kWide);
        RowSum r{m, inv * sum - 1.f, inv * fmaf(-log_own, sum, pull)};
        if (wide || sum < 2.f * own) {
            const int holder = sh.wave[holds].holder;
            float again = 0.f, again_pull = 0.f;
            int ties = 0;
            auto term = [&](float x) __attribute__((always_inline)) {
                float e, d;   // relative to the largest value itself
                if constexpr (KIND == RDK_PROB_F32) {
                    e = x * scale * inv;
                    d = __builtin_amdgcn_logf(fmaxf(e, 0x1p-126f));
                } else {
                    d = fmaxf(a.from_most.of(x, m) * a.from_most.c, -0x1p126f);
                    e = __builtin_amdgcn_exp2f(d);
                    if (x != x) e = x;
                }
                ties += x == m;
                again += x == m ? 0.f : e;
                again_pull = x == m ? again_pull : fmaf(e, d, again_pull);
            };
            // the holder's vectors, or all
            const int stride = wide ? 1 : THREADS, offset = wide ? 0 : holder;
            for (int i = tid; (int64_t)i * stride + offset < whole; i += THREADS) {
                float v[V::kLen];
                V::to(*(const u32x4_any *)(from + ((int64_t)i * stride + offset) * 16), v);
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) term(v[e]);
            }
            if (wide ? tid < behind : tid == 0 && holder < behind) term(load1<KIND>(from, whole * V::kLen + (wide ? tid : holder)));
            again = wave_sum(again);
            again_pull = wave_sum(again_pull);
            ties = wave_count(ties);
            if (lane_id() == 0) {
                sh.others[wid] = again;
                sh.other_pull[wid] = again_pull;
                sh.ties[wid] = ties;
            }
            __syncthreads();
            r.rest = wide ? 0.f : inv * others;
            r.pull = wide ? 0.f : inv * fmaf(-log_own, others, other_pull);
            ties = -1;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                r.rest += sh.others[w];
                r.pull += sh.other_pull[w];
                ties += sh.ties[w];
            }
            r.rest += (float)ties;
        }
        r.pull *= kLn2;
        return r;
    }

    // After finish(): lane c of the first wavefront has what comes before token c in the part.
    __device__ __forceinline__ int counted(const TokenArgs &a, const Shared &sh) const
    {
        int all = count;
        if (RANKS && lane_id() < a.C)
#pragma unroll
            for (int w = 1; w < kWaves; ++w) all += sh.rank[w][lane_id()];
        return all;
    }

    // By the first wavefront: the sums and counts of a part that is one of several.
    __device__ __forceinline__ void write_part(const TokenArgs &a, int64_t row, int part, int parts, RowSum r, const Shared &sh) const
    {
        const int all = counted(a, sh);
        if (lane_id() == 0) a.part_sum[row * parts + part] = make_float4(r.m, r.rest, r.pull, 0.f);
        if (RANKS && lane_id() < a.C) a.part_rank[(row * a.C + lane_id()) * parts + part] = all;
    }
};

// The parts of a row brought together, by one wavefront that writes the row's outputs; all lanes get its sums.  x: the row.
template <int KIND>
__device__ __forceinline__ RowSum merge_tokens(const TokenArgs &a, int64_t row, const void *x, int parts)
{
    const int lane = lane_id();
    int place = kNoToken, count = 0, counts[kMaxTokens];
    float value = no_value<KIND>();
    if (lane < a.C) place = place_of(a.tokens[row * a.C + lane], a.slot_of, a.ids);
    RowSum p{no_value<KIND>(), 0.f, 0.f};
    if (lane < parts) {
        const float4 f = a.part_sum[row * parts + lane];
        p = RowSum{f.x, f.y, f.z};
    }
    if (a.rank) {   // a part to a lane; together on their way
#pragma unroll
        for (int c = 0; c < kMaxTokens; ++c) counts[c] = c < a.C && lane < parts ? a.part_rank[(row * a.C + c) * parts + lane] : 0;
    }
    if (place >= 0) value = load1<KIND>(x, place);
    if (a.rank) {
#pragma unroll
        for (int c = 0; c < kMaxTokens; ++c)
            if (c < a.C) {
                const int all = wave_count(counts[c]);
                if (lane == c) count = all;
            }
    }
    RowSum r;
    r.m = wave_max(p.m);
    const uint64_t who = __ballot(p.m == r.m && p.m > no_value<KIND>());
    const bool holder = who && lane == __ffsll((unsigned long long)who) - 1, none = !(p.m > no_value<KIND>());
    const float far = none ? 0.f : KIND == RDK_PROB_F32 ? logf(p.m / r.m) : a.from_most.of(p.m, r.m) * a.from_most.inv;
    const float f = none ? 0.f : KIND == RDK_PROB_F32 ? p.m / r.m : expf(far), all = f * ((holder ? 0.f : 1.f) + p.rest);
    // (a part without unmasked entries has no terms, but NaN shows in its sum)
    r.rest = wave_sum(none ? p.rest : all);
    r.pull = wave_sum(f == 0.f ? 0.f : fmaf(far, all, f * p.pull));
    write_tokens<KIND>(a, row, r, place, value, count);
    return r;
}

// rdk_logprob.hip: the arguments of a call, and where its parts leave what they come to (returns the bytes)
TokenArgs token_arguments(const rdk_logprobs_desc_t &d, const KernelHandle *h, const int32_t *tokens, float *logprob, int32_t *rank, float *entropy,
                          float4 *stats);
size_t token_places(TokenArgs &t, char *ws, int64_t B, int parts);

// rdk_topk.hip: rows with their top entries
size_t logprobs_top_workspace_bytes(const rdk_logprobs_desc_t &d, rdk_input_kind_t kind);
rdk_status_t launch_logprobs_top(const rdk_logprobs_desc_t &d, RowInput x, TokenArgs t, int32_t *top_ids, float *top_logprobs, void *ws, hipStream_t st);

}  // namespace rdk
