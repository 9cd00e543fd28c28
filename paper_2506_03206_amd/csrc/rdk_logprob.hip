// Log probabilities of given tokens of rows over a vocabulary, their ranks, the row's entropy, and the gradient of these.
//
// With M the row's largest value, Z' the sum over all other entries of exp((x - M) / T) (weights: of x / M) and U the sum of exp((x - M) / T) (x - M) / T:
//   log s_j = (x_j - M) / T - log(1 + Z'),    entropy = log(1 + Z') - U / (1 + Z'),
// every term of which has one sign: a row that is sure of its best entry has an entropy and a log probability of that entry far below
// the rounding of a sum that begins with 1, and they keep their own 24 bits this way.
#include "rdk_select.hpp"
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kMaxTokens = 16;       // given tokens of a row: a lane each
constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kRoundVecs = 4;        // 16-byte vectors of a thread in a round
constexpr int kMaxParts = kWave;     // of a row: a lane each in the finish
constexpr float kLog2e = 1.44269504088896341f;
constexpr double kLn2 = 0.693147180559945309417;

// What a part of a row, or a row, comes to.  m: the largest value; rest: the others' sum relative to it (the largest itself counts 1 beside it);
// pull: the sum of their terms times their distance to it, in units of log e (<= 0).  Of a part without unmasked entries m is none.
struct RowSum {
    float m, rest, pull;
};

struct LogprobArgs {
    const void *x;
    int64_t ldx;
    const int32_t *slot_of;   // target id -> slot, or NULL: ids are places in the row
    const int32_t *kept_ids;  // slot -> target id, with slot_of
    int ids;                  // ids below this are known there
    int n, C, k, parts, part_len;
    float inv_t, c;           // c = log2(e) / T
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *rank;
    int32_t *top_ids;
    float *top;               // values in, log probabilities out
    float4 *stats;            // m, rest, pull / (1 + rest), unused
    float4 *part_sum;         // [B, parts]
    int32_t *part_rank;       // [B, parts, C]
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

// The largest number below x.  (Of -inf, of which nothing is asked, a NaN.)
__device__ __forceinline__ float below(float x)
{
    const uint32_t b = __float_as_uint(x);
    return __uint_as_float(x == 0.f ? 0x80000001u : b + (b >> 31 ? 1u : 0xFFFFFFFFu));
}

// A power of two by which weights up to m come to lie below 2, and its logarithm.  (Weights below 2^-126 stay below 1.)
__device__ __forceinline__ int weight_exponent(float m) { return max((int)(__float_as_uint(m) >> 23) & 0xFF, 1) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }

// The sums that a lane, and later a workgroup, holds: relative to a reference, the largest value not taken out.
//   logits:  ref = largest value;           sum = sum exp((x - ref) / T),   pull = sum exp((x - ref) / T) (x - ref)
//   weights: ref = exponent of the largest; sum = sum w, w = x 2^-ref,      pull = sum w log2 w
template <int KIND>
struct Sums {
    float m, sum, pull;
    float ref, scale;   // (scale: of weights, 2^-ref)

    __device__ __forceinline__ void clear()
    {
        m = no_value<KIND>();
        sum = pull = ref = 0.f;
        scale = 1.f;
    }

    // by what sums change with the reference, and how far it moves (<= 0)
    __device__ __forceinline__ void move(float to, float c)
    {
        const float by = ref - to, f = KIND == RDK_PROB_F32 ? __builtin_amdgcn_exp2f(by) : __builtin_amdgcn_exp2f(by * c);
        pull = sum == 0.f || f == 0.f ? 0.f : f * fmaf(by, sum, pull);
        sum = sum == 0.f ? 0.f : f * sum;
        ref = to;
    }

    __device__ __forceinline__ void raise(float x, float c)
    {
        m = x;
        if constexpr (KIND == RDK_PROB_F32) {
            const float to = (float)weight_exponent(x);
            if (to == ref && sum != 0.f) return;
            move(to, c);
            scale = power_of_two(-(int)to);
        } else {
            move(x, c);
        }
    }

    // (The distance of a masked entry is held finite where 0 multiplies it; NaN is in its term.)
    template <int E>
    __device__ __forceinline__ void add(const float (&x)[E], float c)
    {
        float s = 0.f, p = 0.f;   // a vector's own sums first: long rows are sums of sums
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (KIND == RDK_PROB_F32) {
                const float w = x[i] * scale;
                s += w;
                p = fmaf(w, __builtin_amdgcn_logf(fmaxf(w, 0x1p-126f)), p);   // (log2)
            } else {
                const float d = x[i] - ref, e = __builtin_amdgcn_exp2f(d * c);
                s += e;
                p = fmaf(e, fmaxf(d, -0x1p126f), p);
            }
        }
        sum += s;
        pull += p;
    }
};

struct LogprobShared {
    float wave_m[kWaves], wave_sum[kWaves], wave_pull[kWaves];
    int holder[kWaves];
    int rank[kWaves][kMaxTokens];
    RowSum row;
};

// Sum over the workgroup, the same bits in every thread.  All threads call it.
__device__ __forceinline__ float group_sum(float v, float (&by_wave)[kWaves])
{
    v = wave_sum(v);
    __syncthreads();
    if (lane_id() == 0) by_wave[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += by_wave[w];
    return v;
}

// log probability of an entry x of a row with these sums (logits: m, rest; weights the same)
template <int KIND>
__device__ __forceinline__ float log_share(float x, float m, double log_all, float inv_t)
{
    if (KIND == RDK_PROB_F32) return x > 0.f ? (float)(log((double)x / m) - log_all) : x == 0.f ? -INFINITY : x;
    return x == -INFINITY ? -INFINITY : (float)(((double)x - m) * inv_t - log_all);
}

// The outputs of a row, by one wavefront; count: of lane c, entries before token c.
template <int KIND>
__device__ __forceinline__ void write_tokens(const LogprobArgs &a, int64_t row, RowSum s, int place, float value, int count)
{
    const bool none = s.m == no_value<KIND>() && s.rest == 0.f;
    const double all = 1.0 + (double)s.rest, log_all = log1p((double)s.rest);
    if (lane_id() < a.C) {
        const int64_t o = row * a.C + lane_id();
        float lp = place == kNoToken ? 0.f : -INFINITY;
        if (place >= 0 && !none) lp = log_share<KIND>(value, s.m, log_all, a.inv_t);
        a.logprob[o] = lp;
        if (a.rank) a.rank[o] = place >= 0 && lp > -INFINITY ? count : -1;
    }
    if (lane_id() == 0) {
        const double pull = (double)s.pull / all;
        if (a.entropy) a.entropy[row] = none ? 0.f : (float)(log_all - pull);
        if (a.stats) a.stats[row] = make_float4(s.m, s.rest, (float)pull, 0.f);
    }
}

// Top entries from values to log probabilities, and from slots to ids.
template <int KIND>
__device__ __forceinline__ void write_top(const LogprobArgs &a, int64_t row, RowSum s, int first, int step)
{
    const double log_all = log1p((double)s.rest);
    for (int i = first; i < a.k; i += step) {
        const int64_t o = row * a.k + i;
        const int at = a.top_ids[o];
        a.top[o] = at < 0 ? -INFINITY : log_share<KIND>(a.top[o], s.m, log_all, a.inv_t);
        if (a.kept_ids && at >= 0) a.top_ids[o] = a.kept_ids[at];
    }
}

// One pass over a part of a row.  A lane's sums are relative to the largest value it has seen, so the lane that ends with the largest of all has
// that entry's 1 in its sum, in whose rounding its other entries may be lost; where that matters (all others together come to less than it) this lane's
// vectors are read again, out of the cache, a vector to a thread, and summed without it.  Entries before a token in the order of rdk_topk are those above
// its value, and those that equal it at a lower place: in vectors before its own the bound is the next number below.
template <int KIND>
__global__ __launch_bounds__(kThreads) void logprob_part_kernel(LogprobArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kRound = kThreads * kRoundVecs;   // vectors
    __shared__ LogprobShared sh;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * a.part_len, end = max(begin, min(a.n, begin + a.part_len));
    const int tid = threadIdx.x, wid = tid / kWave;
    const void *xr = row_ptr<KIND>(a.x, a.ldx, row);
    const char *from = (const char *)xr + (int64_t)begin * V::kSize;
    const int whole = (end - begin) / V::kLen, behind = (end - begin) % V::kLen;
    // the tokens, a lane each in every wavefront
    int place = kNoToken, vec = 0;
    float value = no_value<KIND>();
    int count = 0;
    if (lane_id() < a.C) place = place_of(a.tokens[row * a.C + lane_id()], a.slot_of, a.ids);
    if (place >= 0) {
        value = load1<KIND>(xr, place);
        const int here = place - begin;
        vec = here < 0 ? 0 : min(here / V::kLen, whole);
        // equal entries before it in its own vector, which the bounds of vectors pass over (what stands behind the whole vectors is looked at one by one)
        if (a.rank && wid == 0 && here >= 0 && here / V::kLen < whole && here < end - begin)
            for (int e = here / V::kLen * V::kLen; e < here; ++e) count += load1<KIND>(from, e) == value;
    }
    Sums<KIND> s;
    s.clear();
    if (behind > 0 && wid == 0) {
        const float last = tid < behind ? load1<KIND>(from, whole * V::kLen + tid) : no_value<KIND>();
        if (last > s.m) s.raise(last, a.c);
        s.add({last}, a.c);
        if (a.rank)
            for (int c = 0; c < a.C; ++c) {
                const int at = lane_value(place, c);
                const float v = lane_value(value, c);
                const int before = __popcll(__ballot(last > v || (last == v && begin + whole * V::kLen + tid < at)));
                if (lane_id() == c) count += before;
            }
    }
    auto load_round = [&](u32x4 (&raw)[kRoundVecs], int base) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j)
            raw[j] = *(const u32x4_any *)(from + (uint64_t)(uint32_t)min(base + j * kThreads + tid, whole - 1) * 16);
    };
    auto take_round = [&](u32x4 (&now)[kRoundVecs], int base) __attribute__((always_inline)) {
        if (base + kRound > whole) {
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j)
                if (base + j * kThreads + tid >= whole) now[j] = V::fill();
        }
        float vm[kRoundVecs];
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) {
            float v[V::kLen];
            V::to(now[j], v);
            vm[j] = V::largest(v, no_value<KIND>());
            V::again(now[j]);
        }
        static_assert(kRoundVecs == 4, "the largest of a round is formed of four");
        const float most = max3(max3(vm[0], vm[1], vm[2]), vm[3], s.m);
        if (most > s.m) s.raise(most, a.c);
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) {
            float v[V::kLen];
            V::to(now[j], v);
            s.add(v, a.c);
        }
        if (a.rank) {
#pragma unroll 1
            for (int c = 0; c < a.C; ++c) {
                const int at = lane_value(place, c), first = lane_value(vec, c);
                if (at < 0) continue;
                const float v = lane_value(value, c), lower = below(v);
                int all = 0;
#pragma unroll
                for (int j = 0; j < kRoundVecs; ++j) {
                    const float bound = base + j * kThreads + tid < first ? lower : v;
                    if (__ballot(vm[j] > bound)) {
                        float y[V::kLen];
                        V::to(now[j], y);
#pragma unroll
                        for (int e = 0; e < V::kLen; ++e) all += __popcll(__ballot(y[e] > bound));
                    }
                }
                if (lane_id() == c) count += all;
            }
        }
    };
    if (whole > 0) {
        u32x4 raw[kRoundVecs], ahead[kRoundVecs];   // in turn: the round at hand, and the next one on its way
        load_round(raw, 0);
#pragma unroll 1
        for (int base = 0;; base += 2 * kRound) {
            load_round(ahead, base + kRound);
            take_round(raw, base);
            if (base + kRound >= whole) break;
            load_round(raw, base + 2 * kRound);
            take_round(ahead, base + kRound);
            if (base + 2 * kRound >= whole) break;
        }
    }
    // the workgroup's largest value, the first lane that holds it, and the sums relative to it
    const float wave_most = wave_max(s.m);
    if (lane_id() == 0) sh.wave_m[wid] = wave_most;
    if (lane_id() < a.C) sh.rank[wid][lane_id()] = count;
    __syncthreads();
    float m = sh.wave_m[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sh.wave_m[w]);
    const float ref = KIND == RDK_PROB_F32 ? (float)weight_exponent(m) : weight_reference(m);
    if (s.sum != 0.f) s.move(ref, a.c);
    const uint64_t who = __ballot(s.m == m);
    if (lane_id() == 0) sh.holder[wid] = who ? wid * kWave + __ffsll((unsigned long long)who) - 1 : kThreads;
    float sum = group_sum(s.sum, sh.wave_sum), pull = group_sum(s.pull, sh.wave_pull);
    int holder = sh.holder[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) holder = min(holder, sh.holder[w]);
    const float own = KIND == RDK_PROB_F32 ? m * power_of_two(-(int)ref) : 1.f;   // what the largest entry counts
    const bool some = m > no_value<KIND>() && m < INFINITY;
    if (some && sum < 2.f * own && holder < kThreads) {
        Sums<KIND> again;
        again.clear();
        again.ref = ref;
        again.scale = power_of_two(-(int)ref);
        int equal = 0;
        for (int i = tid; i * kThreads + holder < whole; i += kThreads) {
            float v[V::kLen];
            V::to(*(const u32x4_any *)(from + (int64_t)(i * kThreads + holder) * 16), v);
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) {
                equal += v[e] == m;
                v[e] = v[e] == m ? no_value<KIND>() : v[e];
            }
            again.add(v, a.c);
        }
        if (tid == 0 && holder < behind) {
            const float last = load1<KIND>(from, whole * V::kLen + holder);
            equal += last == m;
            again.add({last == m ? no_value<KIND>() : last}, a.c);
        }
        const bool mine = tid == holder;
        const float others = group_sum(again.sum + (mine ? 0.f : s.sum), sh.wave_sum), ties = group_sum((float)equal, sh.wave_m);
        pull = group_sum(again.pull + (mine ? 0.f : s.pull), sh.wave_pull);
        sum = fmaf(ties - 1.f, own, others);
        if constexpr (KIND == RDK_PROB_F32) pull = fmaf((ties - 1.f) * own, __builtin_amdgcn_logf(own), pull);
    } else if (some) {
        sum -= own;
        if constexpr (KIND == RDK_PROB_F32) pull = fmaf(-own, __builtin_amdgcn_logf(own), pull);
    }
    if (wid != 0) {
        if (a.k == 0 || a.parts > 1) return;
    } else {
        RowSum r;
        r.m = m;
        if constexpr (KIND == RDK_PROB_F32) {   // relative to the largest weight itself
            const float inv = 1.f / own;
            r.rest = some ? sum * inv : sum - sum;   // (NaN where there is one, 0 where all is masked)
            r.pull = some ? (float)kLn2 * inv * fmaf(-__builtin_amdgcn_logf(own), sum, pull) : 0.f;
        } else {
            r.rest = some ? sum : sum - sum;
            r.pull = some ? pull * a.inv_t : 0.f;
        }
        if (lane_id() < a.C) {
#pragma unroll
            for (int w = 1; w < kWaves; ++w) count += sh.rank[w][lane_id()];
        }
        if (a.parts > 1) {
            if (lane_id() == 0) a.part_sum[row * a.parts + part] = make_float4(r.m, r.rest, r.pull, 0.f);
            if (a.rank && lane_id() < a.C) a.part_rank[(row * a.parts + part) * a.C + lane_id()] = count;
            return;
        }
        write_tokens<KIND>(a, row, r, place, value, count);
        if (lane_id() == 0) sh.row = r;
    }
    if (a.k == 0) return;
    __syncthreads();
    write_top<KIND>(a, row, sh.row, tid, kThreads);
}

// The parts of a row brought together, by one wavefront.
template <int KIND>
__global__ __launch_bounds__(kWave) void logprob_finish_kernel(LogprobArgs a)
{
    const int64_t row = blockIdx.x;
    const int lane = lane_id();
    RowSum p{no_value<KIND>(), 0.f, 0.f};
    if (lane < a.parts) {
        const float4 f = a.part_sum[row * a.parts + lane];
        p = RowSum{f.x, f.y, f.z};
    }
    int place = kNoToken, count = 0;
    float value = no_value<KIND>();
    if (lane < a.C) {
        place = place_of(a.tokens[row * a.C + lane], a.slot_of, a.ids);
        if (place >= 0) value = load1<KIND>(row_ptr<KIND>(a.x, a.ldx, row), place);
        if (a.rank)
            for (int i = 0; i < a.parts; ++i) count += a.part_rank[(row * a.parts + i) * a.C + lane];
    }
    RowSum r;
    r.m = wave_max(p.m);
    const uint64_t who = __ballot(p.m == r.m && p.m > no_value<KIND>());
    const bool holder = who && lane == __ffsll((unsigned long long)who) - 1, none = !(p.m > no_value<KIND>());
    const double far = none ? 0.0 : KIND == RDK_PROB_F32 ? log((double)p.m / r.m) : ((double)p.m - r.m) * a.inv_t;
    const double f = none ? 0.0 : exp(far), all = f * ((holder ? 0.0 : 1.0) + (double)p.rest);
    // (a part without unmasked entries has no terms, but NaN shows in its sum)
    r.rest = (float)wave_sum(none ? (double)p.rest : all);
    r.pull = (float)wave_sum(f == 0.0 ? 0.0 : fma(far, all, f * (double)p.pull));
    write_tokens<KIND>(a, row, r, place, value, count);
    write_top<KIND>(a, row, r, lane, kWave);
}

// ---- gradient

constexpr int kGradVecs = 8;

struct GradArgs {
    const void *x;
    int64_t ldx;
    const int32_t *slot_of;
    int ids, n, C, parts;
    float inv_t, c, least;    // least: what exponents of base 2 need not go below, over c
    const int32_t *tokens;
    const float4 *stats;
    const float *above, *above_entropy;   // d / d logprob [B, C], d / d entropy [B]; either may be NULL
    void *dx;
    int64_t ldd;
};

// The gradient of a row: dx_j = 1/T (sum of g over the tokens at j - s_j (G + h (log s_j + entropy))), G = sum of g over the tokens that the row holds.
// log s_j + entropy = (x_j - M) / T - pull / (1 + rest): one exponential and two products an element.  At a token of the largest value g - s G is
// (g - G) + G rest / (1 + rest), so that a row that is sure of its token has the gradient that remains.
struct RowGrad {
    float m, c, least, inv_t;
    float a0, a1, G, at_most;

    // stats as LogprobArgs has them
    __device__ __forceinline__ RowGrad(const GradArgs &a, float4 stats, float sum_g, float h) : m(stats.x), c(a.c), least(a.least), inv_t(a.inv_t), G(sum_g)
    {
        const float inv = 1.f / (1.f + stats.y);
        a0 = -inv * inv_t * (G - h * stats.z);
        a1 = -inv * inv_t * (h * inv_t);
        at_most = inv_t * (G * (stats.y * inv) + h * stats.z * inv);   // what remains at the largest value where g = G
    }

    // (The distance of a masked entry is held finite: s = 0, whatever its factor.  NaN is in the row's sum.)
    __device__ __forceinline__ float entry(float x) const
    {
        const float d = fmaxf(x - m, least);
        return __builtin_amdgcn_exp2f(d * c) * fmaf(a1, d, a0);
    }
    __device__ __forceinline__ float token(float x, float y, float g) const { return x == m ? fmaf(g - G, inv_t, at_most) : fmaf(g, inv_t, y); }

    // A lane's vector of the gradient; first: the place of its first entry; place, g: the row's tokens, a lane each.
    template <int KIND>
    __device__ __forceinline__ u32x4 vector(const u32x4 raw, int first, int C, int place, float g) const
    {
        typedef Vec<KIND> V;
        float v[V::kLen], y[V::kLen];
        V::to(raw, v);
#pragma unroll
        for (int e = 0; e < V::kLen; ++e) y[e] = entry(v[e]);
        uint64_t any = 0;
        for (int k = 0; k < C; ++k) any |= __ballot((uint32_t)(lane_value(place, k) - first) < (uint32_t)V::kLen);
        if (any) {
            float add[V::kLen];
            unsigned met = 0;
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) add[e] = 0.f;
            for (int k = 0; k < C; ++k) {
                const int at = lane_value(place, k) - first;
                const float gk = lane_value(g, k);
#pragma unroll
                for (int e = 0; e < V::kLen; ++e)
                    if (at == e) {
                        add[e] += gk;
                        met |= 1u << e;
                    }
            }
#pragma unroll
            for (int e = 0; e < V::kLen; ++e)
                if (met >> e & 1) y[e] = token(v[e], y[e], add[e]);
        }
        return V::from(y);
    }
};

// The gradient of a part of a row, from the statistics that the forward call left.
template <int KIND, int VECS>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(GradArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kSlots = kThreads * VECS * V::kLen;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * kSlots, here = min(a.n - begin, kSlots), tid = threadIdx.x;
    const char *from = (const char *)row_ptr<KIND>(a.x, a.ldx, row) + (int64_t)begin * V::kSize;
    char *to = (char *)const_cast<void *>(row_ptr<KIND>(a.dx, a.ldd, row)) + (int64_t)begin * V::kSize;
    const float h = a.above_entropy ? a.above_entropy[row] : 0.f;
    const float4 st = a.stats[row];
    int place = kNoToken;
    float g = 0.f;
    if (a.above && lane_id() < a.C) {
        place = place_of(a.tokens[row * a.C + lane_id()], a.slot_of, a.ids);
        if (place >= 0) g = a.above[row * a.C + lane_id()];
    }
    const bool masked = st.x == -INFINITY && st.y == 0.f;
    if (masked || (h == 0.f && __ballot(g != 0.f) == 0)) {   // alike for the workgroup: the row is not read
        const u32x4 zero{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            const int left = here - (j * kThreads + tid) * V::kLen;
            if (left > 0) V::store_at(to, (j * kThreads + tid) * 16, left, zero);
        }
        return;
    }
    u32x4 raw[VECS];
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const int left = here - (j * kThreads + tid) * V::kLen;
        raw[j] = left > 0 ? V::load_at(from, (j * kThreads + tid) * 16, left) : V::fill();
    }
    const RowGrad grad(a, st, wave_sum(g), h);
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const int first = (j * kThreads + tid) * V::kLen, left = here - first;
        const u32x4 y = grad.template vector<KIND>(raw[j], begin + first, a.C, place, g);
        if (left > 0) V::store_at(to, first * V::kSize, left, y);
    }
}

// Forward and backward of a row that lies in the registers of one workgroup: read once.
template <int KIND, int THREADS, int VECS>
__global__ __launch_bounds__(THREADS) void logprob_row_kernel(LogprobArgs a, GradArgs b)
{
    typedef Vec<KIND> V;
    constexpr int kW = THREADS / kWave;
    __shared__ float wave_m[kW], wave_rest[kW], wave_pull[kW];
    __shared__ int wave_ties[kW];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, wid = tid / kWave;
    const char *from = (const char *)row_ptr<KIND>(a.x, a.ldx, row);
    u32x4 raw[VECS];
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const int left = a.n - (j * THREADS + tid) * V::kLen;
        raw[j] = left > 0 ? V::load_at(from, (j * THREADS + tid) * 16, left) : V::fill();
    }
    const float h = b.above_entropy ? b.above_entropy[row] : 0.f;
    int place = kNoToken;
    float g = 0.f, value = -INFINITY;
    if (lane_id() < a.C) {
        place = place_of(a.tokens[row * a.C + lane_id()], a.slot_of, a.ids);
        if (place >= 0) {
            value = load1<KIND>(from, place);
            if (b.above) g = b.above[row * a.C + lane_id()];
        }
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        float v[V::kLen];
        V::to(raw[j], v);
        m = V::largest(v, m);
        V::again(raw[j]);
    }
    const float own = wave_max(m);
    if (lane_id() == 0) wave_m[wid] = own;
    asm volatile("" ::"v"(value));   // it is there before another wavefront writes over it (dx may be x)
    __syncthreads();
    m = wave_m[0];
#pragma unroll
    for (int w = 1; w < kW; ++w) m = fmaxf(m, wave_m[w]);
    const float ref = weight_reference(m);
    float rest = 0.f, pull = 0.f;
    int ties = 0;
    if (own == m && m > -INFINITY) {   // a wavefront that holds the largest value: it is left out
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            float v[V::kLen], s = 0.f, p = 0.f;
            V::to(raw[j], v);
            V::again(raw[j]);
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) {
                const float d = v[e] - ref, x = __builtin_amdgcn_exp2f(d * a.c);
                ties += __popcll(__ballot(v[e] == m));
                s += v[e] == m ? 0.f : x;
                p = fmaf(x, fmaxf(d, -0x1p126f), p);
            }
            rest += s;
            pull += p;
        }
    } else {
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            float v[V::kLen], s = 0.f, p = 0.f;
            V::to(raw[j], v);
            V::again(raw[j]);
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) {
                const float d = v[e] - ref, x = __builtin_amdgcn_exp2f(d * a.c);
                s += x;
                p = fmaf(x, fmaxf(d, -0x1p126f), p);
            }
            rest += s;
            pull += p;
        }
    }
    rest = wave_sum(rest);
    pull = wave_sum(pull);
    if (lane_id() == 0) {
        wave_rest[wid] = rest;
        wave_pull[wid] = pull;
        wave_ties[wid] = ties;
    }
    __syncthreads();
    rest = pull = 0.f;
    ties = 0;
#pragma unroll
    for (int w = 0; w < kW; ++w) {
        rest += wave_rest[w];
        pull += wave_pull[w];
        ties += wave_ties[w];
    }
    const bool some = m > -INFINITY && m < INFINITY;
    rest = some ? rest + (float)(ties - 1) : m > 0.f ? NAN : rest - rest;   // (an infinity; NaN where there is one, 0 where all is masked)
    pull = some ? pull * a.inv_t : 0.f;
    const float4 st = make_float4(m, rest, (float)((double)pull / (1.0 + (double)rest)), 0.f);
    if (wid == 0) write_tokens<KIND>(a, row, RowSum{m, rest, pull}, place, value, 0);
    char *to = (char *)const_cast<void *>(row_ptr<KIND>(b.dx, b.ldd, row));
    const bool masked = m == -INFINITY && rest == 0.f;
    if (masked || (h == 0.f && __ballot(g != 0.f) == 0)) {
        const u32x4 zero{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            const int left = a.n - (j * THREADS + tid) * V::kLen;
            if (left > 0) V::store_at(to, (j * THREADS + tid) * 16, left, zero);
        }
        return;
    }
    const RowGrad grad(b, st, wave_sum(g), h);
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const int first = (j * THREADS + tid) * V::kLen, left = a.n - first;
        const u32x4 y = grad.template vector<KIND>(raw[j], first, b.above ? a.C : 0, place, g);
        if (left > 0) V::store_at(to, first * V::kSize, left, y);
    }
}

template <class F>
void with_kind(rdk_input_kind_t kind, const F &f)
{
    if (kind == RDK_PROB_F32) f(std::integral_constant<int, RDK_PROB_F32>());
    else if (kind == RDK_LOGIT_F32) f(std::integral_constant<int, RDK_LOGIT_F32>());
    else f(std::integral_constant<int, RDK_LOGIT_BF16>());
}

struct Parts {
    int count, len;
};
Parts parts_of(int64_t rows, int n, rdk_input_kind_t kind)
{
    const int round = kThreads * kRoundVecs * (kind == RDK_LOGIT_BF16 ? 8 : 4);
    int want = (int)(1024 / rows);
    if (want > kMaxParts) want = kMaxParts;
    if (want <= 1 || n <= 2 * round) return Parts{1, (int)align_up((size_t)n, 64)};
    int64_t len = ((int64_t)n - 1) / want + 1;
    len = (int64_t)align_up((size_t)len, (size_t)(len > round ? round : round / 4));
    return Parts{(int)((n - 1) / len) + 1, (int)len};
}

size_t own_bytes(const rdk_logprobs_desc_t &d, int parts)
{
    if (parts <= 1) return 0;
    return align_up((size_t)d.B * parts * sizeof(float4), 256) + align_up((size_t)d.B * parts * d.C * sizeof(int32_t), 256);
}

rdk_topk_desc_t top_desc(const rdk_logprobs_desc_t &d) { return rdk_topk_desc_t{d.B, d.N, d.k, d.temperature}; }

}  // namespace

int logprobs_max_tokens() { return kMaxTokens; }

size_t logprobs_workspace_bytes(const rdk_logprobs_desc_t &d, rdk_input_kind_t kind)
{
    return align_up((size_t)d.B * sizeof(float4), 256) + own_bytes(d, parts_of(d.B, d.N, kind).count) + (d.k ? topk_workspace_bytes(top_desc(d), kind) : 0);
}

namespace {

LogprobArgs arguments(const rdk_logprobs_desc_t &d, const KernelHandle *h, RowInput x, const int32_t *tokens, float *logprob, int32_t *rank, float *entropy,
                      int32_t *top_ids, float *top_logprobs, float4 *stats, char *ws, Parts split)
{
    LogprobArgs a{};
    a.x = x.ptr; a.ldx = x.ld;
    a.slot_of = h ? h->slot_of : nullptr;
    a.kept_ids = h ? h->kept_ids : nullptr;
    a.ids = h ? h->N : d.N;
    a.n = d.N; a.C = d.C; a.k = d.k; a.parts = split.count; a.part_len = split.len;
    a.inv_t = 1.f / d.temperature;
    a.c = a.inv_t * kLog2e;
    a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.rank = rank;
    a.top_ids = top_ids; a.top = top_logprobs; a.stats = stats;
    a.part_sum = (float4 *)ws;
    a.part_rank = (int32_t *)(ws + align_up((size_t)d.B * split.count * sizeof(float4), 256));
    return a;
}

GradArgs grad_arguments(const rdk_logprobs_desc_t &d, const KernelHandle *h, RowInput x, const int32_t *tokens, const float4 *stats, const float *above,
                        const float *above_entropy, void *dx, int64_t ldd)
{
    GradArgs a{};
    a.x = x.ptr; a.ldx = x.ld;
    a.slot_of = h ? h->slot_of : nullptr;
    a.ids = h ? h->N : d.N;
    a.n = d.N; a.C = d.C;
    a.inv_t = 1.f / d.temperature;
    a.c = a.inv_t * kLog2e;
    const float least = -200.f / a.c;
    a.least = least > -0x1p126f ? least : -0x1p126f;
    a.tokens = tokens; a.stats = stats; a.above = above; a.above_entropy = above_entropy;
    a.dx = dx; a.ldd = ldd;
    return a;
}

template <int KIND>
rdk_status_t launch_rows(const LogprobArgs &a, int32_t B, hipStream_t st)
{
    RDK_TIMED_LAUNCH("logprob_part_kernel", (logprob_part_kernel<KIND>), dim3((unsigned)B * a.parts), dim3(kThreads), 0, st, a);
    if (a.parts > 1) RDK_TIMED_LAUNCH("logprob_finish_kernel", (logprob_finish_kernel<KIND>), dim3((unsigned)B), dim3(kWave), 0, st, a);
    RDK_LAUNCH_CHECK("logprob_part_kernel");
    return RDK_OK;
}

template <int KIND>
rdk_status_t launch_grad(GradArgs a, int32_t B, hipStream_t st)
{
    a.parts = (a.n - 1) / (kThreads * kGradVecs * Vec<KIND>::kLen) + 1;
    RDK_TIMED_LAUNCH("logprob_grad_kernel", (logprob_grad_kernel<KIND, kGradVecs>), dim3((unsigned)B * a.parts), dim3(kThreads), 0, st, a);
    RDK_LAUNCH_CHECK("logprob_grad_kernel");
    return RDK_OK;
}

template <int KIND, int THREADS, int VECS>
rdk_status_t launch_row(const LogprobArgs &a, const GradArgs &b, int32_t B, hipStream_t st)
{
    RDK_TIMED_LAUNCH("logprob_row_kernel", (logprob_row_kernel<KIND, THREADS, VECS>), dim3((unsigned)B), dim3(THREADS), 0, st, a, b);
    RDK_LAUNCH_CHECK("logprob_row_kernel");
    return RDK_OK;
}

template <int KIND>
rdk_status_t launch_step(const LogprobArgs &a, const GradArgs &b, int32_t B, hipStream_t st)
{
    constexpr int kLen = Vec<KIND>::kLen;
    if (a.n <= 256 * 2 * kLen) return launch_row<KIND, 256, 2>(a, b, B, st);
    if (a.n <= 256 * 8 * kLen) return launch_row<KIND, 256, 8>(a, b, B, st);
    if (a.n <= 512 * 8 * kLen) return launch_row<KIND, 512, 8>(a, b, B, st);
    if (a.n <= 512 * 16 * kLen) return launch_row<KIND, 512, 16>(a, b, B, st);
    if (a.n <= 1024 * 16 * kLen) return launch_row<KIND, 1024, 16>(a, b, B, st);
    const rdk_status_t rc = launch_rows<KIND>(a, B, st);
    return rc == RDK_OK ? launch_grad<KIND>(b, B, st) : rc;
}

}  // namespace

rdk_status_t launch_logprobs(const rdk_logprobs_desc_t &d, const KernelHandle *h, RowInput x, const int32_t *tokens, float *logprob, int32_t *rank,
                             float *entropy, int32_t *top_ids, float *top_logprobs, float *stats, void *ws, hipStream_t st)
{
    const Parts split = parts_of(d.B, d.N, x.kind);
    const LogprobArgs a = arguments(d, h, x, tokens, logprob, rank, entropy, top_ids, top_logprobs, (float4 *)stats, (char *)ws, split);
    rdk_status_t rc = RDK_OK;
    if (d.k) rc = launch_topk(top_desc(d), x, top_ids, top_logprobs, nullptr, (char *)ws + own_bytes(d, split.count), st);
    if (rc == RDK_OK) with_kind(x.kind, [&](auto kind) { rc = launch_rows<decltype(kind)::value>(a, d.B, st); });
    return rc;
}

rdk_status_t launch_logprobs_grad(const rdk_logprobs_desc_t &d, const KernelHandle *h, RowInput x, const int32_t *tokens, const float *stats,
                                  const float *above, const float *above_entropy, void *dx, int64_t ldd, hipStream_t st)
{
    const GradArgs a = grad_arguments(d, h, x, tokens, (const float4 *)stats, above, above_entropy, dx, ldd);
    return x.kind == RDK_LOGIT_F32 ? launch_grad<RDK_LOGIT_F32>(a, d.B, st) : launch_grad<RDK_LOGIT_BF16>(a, d.B, st);
}

rdk_status_t launch_logprobs_step(const rdk_logprobs_desc_t &d, const KernelHandle *h, RowInput x, const int32_t *tokens, const float *above,
                                  const float *above_entropy, float *logprob, float *entropy, float *stats, void *dx, int64_t ldd, void *ws,
                                  hipStream_t st)
{
    const Parts split = parts_of(d.B, d.N, x.kind);
    float4 *const kept = stats ? (float4 *)stats : (float4 *)ws;
    const LogprobArgs a = arguments(d, h, x, tokens, logprob, nullptr, entropy, nullptr, nullptr, kept,
                                    (char *)ws + align_up((size_t)d.B * sizeof(float4), 256), split);
    const GradArgs b = grad_arguments(d, h, x, tokens, kept, above, above_entropy, dx, ldd);
    return x.kind == RDK_LOGIT_F32 ? launch_step<RDK_LOGIT_F32>(a, b, d.B, st) : launch_step<RDK_LOGIT_BF16>(a, b, d.B, st);
}

}  // namespace rdk
