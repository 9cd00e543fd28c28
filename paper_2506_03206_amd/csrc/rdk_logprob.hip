// Log probabilities of given tokens of rows over a vocabulary, their ranks, the row's entropy, and the gradient of these.  (With the row's top entries: in
// rdk_topk.hip, in the same pass over the row.)
#include "rdk_tokens.hpp"

namespace rdk {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxParts = kWave;     // of a row: a lane each in the finish
struct LogprobArgs {
    const void *x;
    int64_t ldx;
    int n, parts, part_len;
    TokenArgs t;
};

// One pass over a part of a row; what it sums and counts, and why in that form, stands at TokenPass.  Two rounds of four vectors a thread in turn, one at work
// and one on its way.  Without tokens' ranks it is bound by HBM and by the vector unit in about equal parts (an entry takes some 8 lane operations, an exponential
// of a quarter rate among them): 1024 bf16 rows of 151936 58.5 us = 5.3 TB/s, 2048 fp32 rows of 32064 48 us = 5.5 TB/s; with a token's rank 62.5 and 50.5, and every
// further token 11.5 us (bf16, 155 million entries).  Rows that are all on the chip at once are a chain: loads, sums, two meetings of the wavefronts.
template <int KIND, bool RANKS>
__global__ __launch_bounds__(kThreads) void logprob_part_kernel(LogprobArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kRoundVecs = kTokenRoundVecs, kRound = kThreads * kRoundVecs;   // vectors
    __shared__ TokenShared<kThreads> sh;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * a.part_len, end = max(begin, min(a.n, begin + a.part_len));
    const int tid = threadIdx.x, wid = tid / kWave;
    const void *xr = row_ptr<KIND>(a.x, a.ldx, row);
    const char *from = (const char *)xr + (int64_t)begin * V::kSize;
    const int whole = (end - begin) / V::kLen, behind = (end - begin) % V::kLen;
    TokenPass<KIND, kThreads, RANKS> pass;
    // Always as many loads, of the last vector where the round has none of its own: the compiler counts loads in flight, and would wait for all of
    // them behind a branch that has some of its own.
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
        for (int j = 0; j < kRoundVecs; ++j) vm[j] = pass.vector(a.t, now[j]);
        static_assert(kRoundVecs == 4, "the largest of a round is formed of four");
        const float most = max3(max3(vm[0], vm[1], vm[2]), vm[3], no_value<KIND>());
        pass.s.m = fmaxf(pass.s.m, most);
        if constexpr (RANKS) pass.ranks(a.t, now, most, base);
    };
    u32x4 raw[kRoundVecs], ahead[kRoundVecs];   // in turn: the round at hand, and the next one on its way
    if (whole > 0) load_round(raw, 0);
    pass.begin(a.t, row, xr, begin, begin + whole * V::kLen, a.n);
    if (behind > 0 && wid == 0)
        pass.single(a.t, tid < behind ? load1<KIND>(from, whole * V::kLen + tid) : no_value<KIND>(), begin + whole * V::kLen + tid);
    if (whole > 0) {
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
    const RowSum r = pass.finish(a.t, from, whole, behind, sh);
    if (wid != 0) return;
    if (a.parts > 1) pass.write_part(a.t, row, part, a.parts, r, sh);
    else write_tokens<KIND>(a.t, row, r, pass.place, pass.value, pass.counted(a.t, sh));
}

// The parts of a row brought together, by one wavefront: a chain of a read, a dozen exchanges between lanes and a write, 2.4 to 3.4 us.
template <int KIND>
__global__ __launch_bounds__(kWave) void logprob_finish_kernel(LogprobArgs a)
{
    const int64_t row = blockIdx.x;
    merge_tokens<KIND>(a.t, row, row_ptr<KIND>(a.x, a.ldx, row), a.parts);
}

// ---- gradient

constexpr int kGradVecs = 8;

struct GradArgs {
    const void *x;
    int64_t ldx;
    const int32_t *slot_of;
    int ids, n, C, parts;
    float inv_t;
    Distance from_most;
    float least;              // what distances need not go below: 200 in units of log 2
    const int32_t *tokens;
    const float4 *stats;
    const float *above, *above_entropy;   // d / d logprob [B, C], d / d entropy [B]; either may be NULL
    void *dx;
    int64_t ldd;
};

// The gradient of a row: dx_j = 1/T (sum of g over the tokens at j - s_j (G + h (log s_j + entropy))), G = sum of g over the tokens that the row holds.
// log s_j + entropy = (x_j - M) / T - pull / (1 + rest): one exponential and two products an element, with distances in units of about T (the square of 1 / T in the
// entropy's term would be 0 at high temperatures).  At tokens of the largest value, where s = 1 / (1 + rest), g - s G is
// g rest / (1 + rest) - s (sum of g over the row's other tokens): no difference of g and G, of which nothing is left where the row is sure of its only token (rest far below
// 2^-24), and beside whose rounding s is nothing where the row is flat.
struct RowGrad {
    float m, least, inv_t;
    Distance from_most;
    float a0, a1, s_most, q_most, h_most;   // of the largest value: s, rest / (1 + rest), and what the entropy adds before 1 / T

    // stats as TokenArgs has them
    __device__ __forceinline__ RowGrad(const GradArgs &a, float4 stats, float G, float h) : m(lane_value(stats.x, 0)), least(a.least), inv_t(a.inv_t), from_most(a.from_most)
    {
        const float inv = 1.f / (1.f + stats.y);   // (all of it is alike for the wavefront: scalar registers)
        a0 = lane_value(-(inv * (G - h * stats.z)) * inv_t, 0);
        a1 = lane_value(-(inv * (h * from_most.inv)) * inv_t, 0);
        s_most = lane_value(inv, 0);
        q_most = lane_value(stats.y * inv, 0);
        h_most = lane_value(h * stats.z * inv, 0);
    }

    // A lane's vector of the gradient; first: the place of its first entry; place, g, elsewhere: the row's tokens, a lane each, and the sum of g over tokens at other
    // places; terms: exp((x - M) / T) of its entries.
    template <int KIND>
    __device__ __forceinline__ u32x4 vector(const u32x4 raw, const float (&terms)[Vec<KIND>::kLen], int first, int C, int place, float g, float elsewhere) const
    {
        typedef Vec<KIND> V;
        float v[V::kLen], y[V::kLen];
        V::to(raw, v);
        if (a1 == 0.f) {
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) y[e] = terms[e] * a0;
        } else {   // (The distance of a masked entry is held finite: s = 0, whatever its factor.  NaN is in the row's sum.)
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) y[e] = terms[e] * fmaf(a1, fmaxf(from_most.of(v[e], m), least), a0);
        }
        uint64_t any = 0;
        for (int k = 0; k < C; ++k) any |= __ballot((uint32_t)(lane_value(place, k) - first) < (uint32_t)V::kLen);
        if (any) {
            unsigned most = 0;   // entries of the largest value that tokens have met: before 1 / T
            for (int k = 0; k < C; ++k) {
                const int at = lane_value(place, k) - first;
                if (__ballot((uint32_t)at < (uint32_t)V::kLen) == 0) continue;
                const float gk = lane_value(g, k), others = lane_value(elsewhere, k);
#pragma unroll
                for (int e = 0; e < V::kLen; ++e)
                    if (at == e) {
                        if (v[e] == m) {
                            if (!(most >> e & 1)) y[e] = fmaf(-others, s_most, h_most);
                            y[e] = fmaf(gk, q_most, y[e]);
                            most |= 1u << e;
                        } else {
                            y[e] = fmaf(gk, inv_t, y[e]);
                        }
                    }
            }
#pragma unroll
            for (int e = 0; e < V::kLen; ++e)
                if (most >> e & 1) y[e] *= inv_t;
        }
        return V::from(y);
    }
    template <int KIND>
    __device__ __forceinline__ u32x4 vector(const u32x4 raw, int first, int C, int place, float g, float elsewhere) const
    {
        float v[Vec<KIND>::kLen];
        Vec<KIND>::to(raw, v);
#pragma unroll
        for (int e = 0; e < Vec<KIND>::kLen; ++e) v[e] = __builtin_amdgcn_exp2f(from_most.of(v[e], m) * from_most.c);
        return vector<KIND>(raw, v, first, C, place, g, elsewhere);
    }
};

// In lane c: the sum of g over the tokens that lie at other places than token c.  (g is 0 of those that the row does not hold.)
__device__ __forceinline__ float tokens_elsewhere(int place, float g, int C)
{
    float sum = 0.f;
    for (int k = 0; k < C; ++k) {
        const float gk = lane_value(g, k);
        sum += lane_value(place, k) != place ? gk : 0.f;
    }
    return sum;
}

// The gradient of a part of a row, from the statistics that the forward call left.  One exponential and two or three products an entry, nothing to meet for: HBM
// (2048 fp32 rows of 32064 95 us = 5.5 TB/s read and written), or the last-level cache where the logits still lie there (1024 bf16 rows of 16384 9.6-11.7 us = 5.7 TB/s
// and above).  Rows of which nothing is asked are set to 0 without being read.
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
    const float elsewhere = tokens_elsewhere(place, g, a.C);
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const int first = (j * kThreads + tid) * V::kLen, left = here - first;
        const u32x4 y = grad.template vector<KIND>(raw[j], begin + first, a.C, place, g, elsewhere);
        if (left > 0) V::store_at(to, first * V::kSize, left, y);
    }
}

// Forward and backward of a row that lies in the registers of one workgroup, or forward alone (GRAD, RANKS: which): read once.  The largest value is known before
// the first exponential, so sums need no second reference and what the largest leaves out is left out at once.  With two vectors a thread the exponentials are kept
// for the gradient; with more they are formed again, because registers decide how many rows lie beside each other (2048 bf16 rows of 32064, 512 threads of eight
// vectors: 55 us with 5 wavefronts a SIMD unit, 60 with 6, which spill, 67 with exponentials kept).  HBM: 2048 rows of 32064 52.5 us = 5.0 TB/s read and written,
// fp32 97 us = 5.4 TB/s.
template <int KIND, int THREADS, int VECS, bool GRAD, bool RANKS>
__global__ __launch_bounds__(THREADS, VECS <= 8 ? 5 : 4) void logprob_row_kernel(LogprobArgs a, GradArgs b)
{
    typedef Vec<KIND> V;
    constexpr int kW = THREADS / kWave;
    constexpr bool kKeep = GRAD && VECS <= 2;
    // g asked for behind the sums, where registers are short while they run (16 vectors: 8 registers spilled become 1, 1024 rows of 60000 54.5 -> 49.3 us; eight 48 -> 51 and so not)
    constexpr bool kLate = VECS > 8;
    __shared__ float wave_m[kW], wave_rest[kW], wave_pull[kW];
    __shared__ int wave_ties[kW], wave_rank[RANKS ? kW : 1][kMaxTokens];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, wid = tid / kWave;
    const char *from = (const char *)row_ptr<KIND>(a.x, a.ldx, row);
    // whole vectors; a vector that is not whole behind them is one thread's
    const int whole = a.n / V::kLen, behind = a.n % V::kLen, last_tid = whole % THREADS, last_vec = whole / THREADS;
    u32x4 raw[VECS], last = V::fill();
    if (whole > 0) {
#pragma unroll
        for (int j = 0; j < VECS; ++j) raw[j] = *(const u32x4_any *)(from + (uint32_t)min(j * THREADS + tid, whole - 1) * 16u);
    }
    if (behind > 0 && tid == last_tid) last = V::load_at(from, (uint32_t)whole * 16u, behind);
    const float h = GRAD && b.above_entropy ? b.above_entropy[row] : 0.f;
    int place = kNoToken, count = 0;
    float g = 0.f, value = RANKS ? NAN : -INFINITY;   // (nothing is before none)
    if (lane_id() < a.t.C) {
        place = place_of(a.t.tokens[row * a.t.C + lane_id()], a.t.slot_of, a.t.ids);
        if (place >= 0) {
            value = load1<KIND>(from, place);
            if (GRAD && !kLate && b.above) g = b.above[row * a.t.C + lane_id()];
            if (RANKS && wid == 0) {   // entries of its own vector that equal it and lie before it
                const int own = place & ~(V::kLen - 1);
                float v[V::kLen];
                V::to(V::load(from, own, a.n), v);
#pragma unroll
                for (int e = 0; e < V::kLen - 1; ++e) count += (own + e < place) & (v[e] == value);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < VECS; ++j)
        if (j * THREADS + tid >= whole) raw[j] = j == last_vec ? last : V::fill();   // (fill but for one thread)
    float m = no_value<KIND>();
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        float v[V::kLen];
        V::to(raw[j], v);
        m = V::largest(v, m);
        V::again(raw[j]);
        __builtin_amdgcn_sched_barrier(0);
    }
    const float own = wave_max(m);
    if (lane_id() == 0) wave_m[wid] = own;
    if (GRAD) asm volatile("" ::"v"(value));   // it is there before another wavefront writes over it (dx may be x)
    __syncthreads();
    m = wave_m[0];
#pragma unroll
    for (int w = 1; w < kW; ++w) m = fmaxf(m, wave_m[w]);
    const float ref = weight_reference(m);
    // (Values from `far` on lie 2^103 T apart: all but the largest, which the sums leave out, are then held to be infinitely far.)
    const float minus_ref = fabsf(ref) < a.t.far ? -ref * a.t.in_sums.unit : -INFINITY;
    // of weights: a power of two that keeps them from overflowing and from having few bits, and the largest's reciprocal beside it
    const float scale = KIND == RDK_PROB_F32 ? power_of_two(-weight_exponent(m)) : 1.f, inv = KIND == RDK_PROB_F32 ? m > 0.f ? 1.f / (m * scale) : 0.f : 1.f;
    // an entry relative to the largest value, and its distance from it: in the units of in_sums, of log 2 for weights
    auto term = [&](float v, float &d) __attribute__((always_inline)) {
        if constexpr (KIND == RDK_PROB_F32) {
            const float x = v * scale * inv;
            d = __builtin_amdgcn_logf(fmaxf(x, 0x1p-126f));
            return x;
        } else {
            d = fmaf(v, a.t.in_sums.unit, minus_ref);
            return __builtin_amdgcn_exp2f(d * a.t.in_sums.c);
        }
    };
    float rest = 0.f, pull = 0.f, terms[kKeep ? VECS : 1][V::kLen];
    int ties = 0;
    const bool holds = own == m && m > no_value<KIND>();   // a wavefront that holds the largest value: that is left out
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        float v[V::kLen], s = 0.f, p = 0.f;
        V::to(raw[j], v);
        V::again(raw[j]);
#pragma unroll
        for (int e = 0; e < V::kLen; ++e) {
            float d;
            const float x = term(v[e], d);
            if constexpr (kKeep) terms[j][e] = x;
            s += x;
            p = fmaf(x, d, p);
        }
        if (KIND != RDK_PROB_F32 && p != p) {   // 0 times the distance of a masked entry: such distances are held finite.  (NaN is in the sum.)
            p = 0.f;
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) {
                float d;
                const float x = term(v[e], d);
                p = fmaf(x, fmaxf(d, -0x1p126f), p);
            }
        }
        if (holds) {
            float most = V::largest(v, no_value<KIND>());
            if (__ballot(most == m)) {   // (of a logit the distance is 0; of a weight a product that may be rounded, so it is left out of both)
                s = 0.f;
                if (KIND == RDK_PROB_F32) p = 0.f;
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) {
                    float d;
                    const float x = term(v[e], d);
                    ties += __popcll(__ballot(v[e] == m));
                    s += v[e] == m ? 0.f : x;
                    if constexpr (kKeep) terms[j][e] = v[e] == m ? 1.f : x;
                    if (KIND == RDK_PROB_F32) p = v[e] == m ? p : fmaf(x, d, p);
                }
            }
        }
        rest += s;
        pull += p;
        __builtin_amdgcn_sched_barrier(0);   // (one vector after the other, or registers hold fewer workgroups)
    }
    rest = wave_sum(rest);
    pull = wave_sum(pull);
    if (lane_id() == 0) {
        wave_rest[wid] = rest;
        wave_pull[wid] = pull;
        wave_ties[wid] = ties;
    }
    if (GRAD && kLate && b.above && place >= 0) g = b.above[row * a.t.C + lane_id()];
    if constexpr (RANKS) {
#pragma unroll 1
        for (int c = 0; c < a.t.C; ++c) {
            const float v = lane_value(value, c);
            if (!(own >= v)) continue;   // (alike for the wavefront)
            const int all = wave_count((int)entries_before<KIND, THREADS>(raw, 0, lane_value(place, c) / V::kLen, v));
            if (lane_id() == c) count += all;
        }
        if (lane_id() < a.t.C) wave_rank[wid][lane_id()] = count;
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
    const bool some = m > no_value<KIND>() && m < INFINITY;
    rest = some ? rest + (float)(ties - 1) : m > 0.f ? NAN : rest - rest;   // (an infinity; NaN where there is one, 0 where all is masked)
    pull = some ? pull * (KIND == RDK_PROB_F32 ? kLn2 : a.t.in_sums.inv) : 0.f;
    const float4 st = make_float4(m, rest, pull / (1.f + rest), 0.f);
    if (wid == 0) {
        if (RANKS && lane_id() < a.t.C)
#pragma unroll
            for (int w = 1; w < kW; ++w) count += wave_rank[w][lane_id()];
        write_tokens<KIND>(a.t, row, RowSum{m, rest, pull}, place, value, count);
    }
    if constexpr (GRAD) {
        char *to = (char *)const_cast<void *>(row_ptr<KIND>(b.dx, b.ldd, row));
        const bool masked = m == -INFINITY && rest == 0.f;
        if (masked || (h == 0.f && __ballot(g != 0.f) == 0)) {
            const u32x4 zero{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < VECS; ++j)
                if (j * THREADS + tid < whole) V::store_at(to, (uint32_t)(j * THREADS + tid) * 16u, V::kLen, zero);
            if (behind > 0 && tid == last_tid) V::store_at(to, (uint32_t)whole * 16u, behind, zero);
            return;
        }
        const RowGrad grad(b, st, wave_sum(g), h);
        const int C = b.above ? b.C : 0;
        const float elsewhere = tokens_elsewhere(place, g, C);
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            const int at = j * THREADS + tid;
            u32x4 y;
            if constexpr (kKeep) y = grad.template vector<KIND>(raw[j], terms[j], at * V::kLen, C, place, g, elsewhere);
            else y = grad.template vector<KIND>(raw[j], at * V::kLen, C, place, g, elsewhere);
            if (at < whole) V::store_at(to, (uint32_t)at * 16u, V::kLen, y);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (behind > 0 && wid == last_tid / kWave) {
            const u32x4 y = grad.template vector<KIND>(last, whole * V::kLen - (last_tid - tid) * V::kLen, C, place, g, elsewhere);
            if (tid == last_tid) V::store_at(to, (uint32_t)whole * 16u, behind, y);
        }
    }
}

// Parts of a row: as many workgroups as fill the chip four times, each of a whole round at least.
struct Parts {
    int count, len;
};
Parts parts_of(int64_t rows, int n, rdk_input_kind_t kind)
{
    const int round = kThreads * kTokenRoundVecs * (kind == RDK_LOGIT_BF16 ? 8 : 4);
    int want = (int)(1024 / rows);
    if (want > kMaxParts) want = kMaxParts;
    if (want <= 1 || n <= 2 * round) return Parts{1, (int)align_up((size_t)n, 64)};
    int64_t len = ((int64_t)n - 1) / want + 1;
    len = (int64_t)align_up((size_t)len, (size_t)(len > round ? round : round / 4));
    return Parts{(int)((n - 1) / len) + 1, (int)len};
}

LogprobArgs arguments(const rdk_logprobs_desc_t &d, RowInput x, const TokenArgs &t, char *ws)
{
    const Parts split = parts_of(d.B, d.N, x.kind);
    LogprobArgs a{};
    a.x = x.ptr; a.ldx = x.ld;
    a.n = d.N; a.parts = split.count; a.part_len = split.len;
    a.t = t;
    token_places(a.t, ws, d.B, split.count);
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
    a.from_most = Distance::over(d.temperature);
    a.inv_t = a.from_most.inv * a.from_most.unit;
    const float least = -200.f / a.from_most.c;
    a.least = least > -0x1p126f ? least : -0x1p126f;
    a.tokens = tokens; a.stats = stats; a.above = above; a.above_entropy = above_entropy;
    a.dx = dx; a.ldd = ldd;
    return a;
}

template <int KIND>
rdk_status_t launch_rows(const LogprobArgs &a, int32_t B, hipStream_t st)
{
    const dim3 grid((unsigned)B * a.parts), block(kThreads);
    if (a.t.rank) RDK_TIMED_LAUNCH("logprob_part_kernel", (logprob_part_kernel<KIND, true>), grid, block, before_tokens_bytes(a.t, kThreads), st, a);
    else RDK_TIMED_LAUNCH("logprob_part_kernel", (logprob_part_kernel<KIND, false>), grid, block, 0, st, a);
    if (a.parts > 1) RDK_TIMED_LAUNCH("logprob_finish_kernel", (logprob_finish_kernel<KIND>), dim3((unsigned)B), dim3(kWave), 0, st, a);
    RDK_LAUNCH_CHECK("logprob_part_kernel");
    return RDK_OK;
}

template <int KIND>
rdk_status_t launch_grad(GradArgs a, int32_t B, hipStream_t st)
{
    a.parts = logprobs_grad_parts(a.n, (rdk_input_kind_t)KIND);
    // (a thread asks for no more vectors than short rows have: 8192 bf16 rows of 4096 33.2 -> 21.8 us)
    if (a.n <= kThreads * 2 * Vec<KIND>::kLen)
        RDK_TIMED_LAUNCH("logprob_grad_kernel", (logprob_grad_kernel<KIND, 2>), dim3((unsigned)B), dim3(kThreads), 0, st, a);
    else
        RDK_TIMED_LAUNCH("logprob_grad_kernel", (logprob_grad_kernel<KIND, kGradVecs>), dim3((unsigned)B * a.parts), dim3(kThreads), 0, st, a);
    RDK_LAUNCH_CHECK("logprob_grad_kernel");
    return RDK_OK;
}

template <int KIND, int THREADS, int VECS, bool GRAD = true>
rdk_status_t launch_row(const LogprobArgs &a, const GradArgs &b, int32_t B, hipStream_t st)
{
    const dim3 grid((unsigned)B), block(THREADS);
    if constexpr (GRAD) {
        RDK_TIMED_LAUNCH("logprob_row_kernel", (logprob_row_kernel<KIND, THREADS, VECS, true, false>), grid, block, 0, st, a, b);
    } else {
        if (a.t.rank) RDK_TIMED_LAUNCH("logprob_row_kernel", (logprob_row_kernel<KIND, THREADS, VECS, false, true>), grid, block, 0, st, a, b);
        else RDK_TIMED_LAUNCH("logprob_row_kernel", (logprob_row_kernel<KIND, THREADS, VECS, false, false>), grid, block, 0, st, a, b);
    }
    RDK_LAUNCH_CHECK("logprob_row_kernel");
    return RDK_OK;
}

// The forward call.  Rows that the registers of a workgroup hold take one launch and one look at their largest value, which is known before the first exponential (with a
// token's rank, in rounds or parts -> this way: 8192 bf16 rows of 4096 42.8 -> 21.0 us, 2048 of 1000 13.4 -> 7.1, 1024 of 16384 13.5 -> 12.7, 2048 of 32064 32.3 -> 30.9, 64 of
// 32064 12.5 -> 6.5, 8192 fp32 rows of 2048 33.6 -> 16.2).  Weights take more registers: 512 rows of 16384 14.2 -> 10.2, 1024 16.2 -> 17.3 and so not.  1024 threads where a
// row has a compute unit for itself (256 bf16 rows of 65536 16.0 -> 12.9, 512 21.2 -> 23.3; 256 rows of 32000 weights, 8 tokens 19.6 -> 14.8); a few rows of many tokens
// are spread over more units instead, whose wavefronts have fewer ranks to count (bf16 rows of 65536, this way / in parts: 31 rows with one token 9.3 / 12.5, with two 10.6 / 13.1,
// three 11.8 / 13.7, eight 18.3 / 17.7, 32 rows the same; 8 rows with two 10.4 / 10.6, three 11.7 / 10.5, eight 18.1 / 12.2; so the line at 32 rows gives up to 2 us of three or four
// tokens away, and of fp32 rows, which come out ahead this way up to eight tokens from 24 rows on, up to 3: 31 of 32768, three tokens 8.2 / 11.2).  A launch counts its threads in 32
// bits.
template <int KIND>
rdk_status_t launch_forward(const LogprobArgs &a, int32_t B, hipStream_t st)
{
    constexpr int kLen = Vec<KIND>::kLen;
    const GradArgs none{};
    if (a.n <= 256 * 2 * kLen) return launch_row<KIND, 256, 2, false>(a, none, B, st);
    if (a.n <= 256 * 4 * kLen) return launch_row<KIND, 256, 4, false>(a, none, B, st);
    if (a.n <= 256 * 8 * kLen) return launch_row<KIND, 256, 8, false>(a, none, B, st);
    if (a.n <= 512 * 8 * kLen && (KIND != RDK_PROB_F32 ? B < (1 << 23) : B <= 512)) return launch_row<KIND, 512, 8, false>(a, none, B, st);
    if (a.n <= 1024 * 8 * kLen && B <= 256 && (B >= 32 || a.t.C <= 2)) return launch_row<KIND, 1024, 8, false>(a, none, B, st);
    return launch_rows<KIND>(a, B, st);
}

template <int KIND>
rdk_status_t launch_step(const LogprobArgs &a, const GradArgs &b, int32_t B, hipStream_t st)
{
    constexpr int kLen = Vec<KIND>::kLen;
    // Few long rows: several workgroups to a row, in one launch or two more (bf16: 16 rows of 128256 20.3 -> 15.9 us, 128 of 32064 8.4 in one launch, 512 of
    // 128256 62 in one and 73 in three).
    if (a.parts > 1 && B < 128 && a.n > 512 * 8 * kLen) {
        const rdk_status_t rc = launch_forward<KIND>(a, B, st);
        return rc == RDK_OK ? launch_grad<KIND>(b, B, st) : rc;
    }
    if (a.n <= 256 * 2 * kLen) return launch_row<KIND, 256, 2>(a, b, B, st);
    if (a.n <= 256 * 8 * kLen) return launch_row<KIND, 256, 8>(a, b, B, st);
    if (a.n <= 512 * 8 * kLen) return launch_row<KIND, 512, 8>(a, b, B, st);
    if (a.n <= 512 * 16 * kLen) return launch_row<KIND, 512, 16>(a, b, B, st);
    if (a.n <= 1024 * 16 * kLen) return launch_row<KIND, 1024, 16>(a, b, B, st);
    const rdk_status_t rc = launch_rows<KIND>(a, B, st);
    return rc == RDK_OK ? launch_grad<KIND>(b, B, st) : rc;
}

}  // namespace

int logprobs_max_tokens() { return kMaxTokens; }

int logprobs_grad_parts(int32_t N, rdk_input_kind_t kind)
{
    return (N - 1) / (kThreads * kGradVecs * (kind == RDK_LOGIT_BF16 ? 8 : 4)) + 1;
}

TokenArgs token_arguments(const rdk_logprobs_desc_t &d, const KernelHandle *h, const int32_t *tokens, float *logprob, int32_t *rank, float *entropy,
                          float4 *stats)
{
    TokenArgs t{};
    t.slot_of = h ? h->slot_of : nullptr;
    t.kept_ids = h ? h->kept_ids : nullptr;
    t.ids = h ? h->N : d.N;
    t.C = d.C;
    t.from_most = Distance::over(d.temperature);
    t.in_sums = Distance::in_sums(d.temperature);
    t.far = t.in_sums.unit > 1.f ? 0x1p126f / t.in_sums.unit : INFINITY;
    t.c = t.from_most.c * t.from_most.unit;
    t.margin = 8.f / t.c;
    t.tokens = tokens; t.logprob = logprob; t.entropy = entropy; t.rank = rank; t.stats = stats;
    return t;
}

size_t token_places(TokenArgs &t, char *ws, int64_t B, int parts)
{
    if (parts <= 1) return 0;
    const size_t sums = align_up((size_t)B * parts * sizeof(float4), 256);
    t.part_sum = (float4 *)ws;
    t.part_rank = (int32_t *)(ws + sums);
    return sums + align_up((size_t)B * parts * t.C * sizeof(int32_t), 256);
}

// The statistics of a step that keeps them for itself, then what the parts leave.
size_t logprobs_workspace_bytes(const rdk_logprobs_desc_t &d, rdk_input_kind_t kind)
{
    if (d.k > 0) return logprobs_top_workspace_bytes(d, kind);
    TokenArgs t{};
    t.C = d.C;
    return align_up((size_t)d.B * sizeof(float4), 256) + token_places(t, nullptr, d.B, parts_of(d.B, d.N, kind).count);
}

rdk_status_t launch_logprobs(const rdk_logprobs_desc_t &d, const KernelHandle *h, RowInput x, const int32_t *tokens, float *logprob, int32_t *rank,
                             float *entropy, int32_t *top_ids, float *top_logprobs, float *stats, void *ws, hipStream_t st)
{
    const TokenArgs t = token_arguments(d, h, tokens, logprob, rank, entropy, (float4 *)stats);
    if (d.k > 0) return launch_logprobs_top(d, x, t, top_ids, top_logprobs, ws, st);
    const LogprobArgs a = arguments(d, x, t, (char *)ws);
    if (x.kind == RDK_PROB_F32) return launch_forward<RDK_PROB_F32>(a, d.B, st);
    return x.kind == RDK_LOGIT_F32 ? launch_forward<RDK_LOGIT_F32>(a, d.B, st) : launch_forward<RDK_LOGIT_BF16>(a, d.B, st);
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
    float4 *const kept = stats ? (float4 *)stats : (float4 *)ws;
    const TokenArgs t = token_arguments(d, h, tokens, logprob, nullptr, entropy, kept);
    const LogprobArgs a = arguments(d, x, t, (char *)ws + align_up((size_t)d.B * sizeof(float4), 256));
    const GradArgs b = grad_arguments(d, h, x, tokens, kept, above, above_entropy, dx, ldd);
    return x.kind == RDK_LOGIT_F32 ? launch_step<RDK_LOGIT_F32>(a, b, d.B, st) : launch_step<RDK_LOGIT_BF16>(a, b, d.B, st);
}

}  // namespace rdk
