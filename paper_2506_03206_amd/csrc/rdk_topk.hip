// The k largest entries of rows over a vocabulary with the logarithm of their normaliser, and beam search's selection over beams and
// vocabulary, which takes the K largest entries of every live beam and merges them per request.  The log probabilities of given tokens with the row's top
// entries beside them come from the same pass.
#include "rdk_tokens.hpp"

namespace rdk {

namespace {

constexpr int kTopThreads = 256;

constexpr int kRoundVecs = 4;          // 16-byte vectors of a lane in a round
constexpr int kNoted = 512, kFound = 1024;   // vectors noted by a wavefront, entries sorted: what exceeds these takes a slower way
constexpr int kSift = 4;               // noted vectors read at a time
constexpr int kMergeEntries = 4096;    // of a row's parts together
constexpr int kBeamEntries = 16384;    // of a request's beams and their parts together
constexpr int kTopWaves = kTopThreads / kWave;

struct TopArgs {
    const void *x;
    int64_t ldx;
    int N, k, parts, part_len;
    float inv_t, c;         // c = log2(e) / temperature
    float limit, margin;    // rows of logits with a maximum beyond +-limit are summed anew; 60 / c
    // rows of beams that have no candidates among the ids are passed over
    const float *scores;
    const uint8_t *finished;
    int W;                  // rows that are merged: the beams of a request, 1 otherwise
    uint64_t *entries;      // [rows / W, k, parts, W], 0 where a part has fewer; or NULL: the outputs of topk itself
    SoftStat *stat;         // [rows, parts]
    int32_t *ids;
    float *values, *lse;
};

struct NoTokens {};

struct TopShared {
    SelectShared slow;
    uint64_t found[kFound];
    float2 queue[kTopWaves][kNoted];   // of a wavefront's vectors: the largest value and the place
    int noted[kTopWaves];
    float wave_m[kTopWaves], wave_s[kTopWaves], bound[kTopWaves];
    int count;
};

// What a pass over tokens keeps in LDS, of the kernels that make one.
template <bool TOKENS>
__device__ __forceinline__ TokenShared<kTopThreads> &token_shared()
{
    __shared__ TokenShared<kTopThreads> sh;
    return sh;
}

// The nth largest of the keys of 64 lanes, to their highest BITS bits, by halving.  (Rolled up: code that runs once is fetched while it runs.)
template <int BITS>
__device__ __forceinline__ uint32_t wave_nth(uint32_t key, int nth)
{
    key >>= 32 - BITS;
    uint32_t found = 0;
#pragma unroll 4
    for (int bit = BITS - 1; bit >= 0; --bit) {
        const uint32_t tried = found | (1u << bit);
        if (__popcll(__ballot(key >= tried)) >= nth) found = tried;
    }
    return found << (32 - BITS);
}

// A value that no entry that is wanted lies below: the nth largest of the lanes' largest values, to the highest BITS bits of its key (sixteen are all
// that a bf16 value has).  With fewer lanes that have unmasked values: every unmasked value is wanted.
template <int KIND, int BITS>
__device__ __forceinline__ float wave_bound(float largest, int nth)
{
    const uint32_t key = wave_nth<BITS>(order_key(largest), nth);
    if (key <= masked_key<KIND>()) return KIND == RDK_PROB_F32 ? __uint_as_float(1u) : -3.402823466e38f;
    return key_value(KIND == RDK_LOGIT_BF16 && !(key >> 31) ? key | 0xFFFFu : key);   // (the key of a negative bf16 value ends in ones)
}

// The sum of exp((x - m) / T) over a part, for a largest value m so far from zero that the rounding of its product with 1 / T is no small number.
template <int KIND>
__device__ __forceinline__ float wide_sum(const TopArgs &a, const void *xr, int begin, int end, float m, TopShared &sh)
{
    float s = 0.f;
    for (int i = begin + (int)threadIdx.x; i < end; i += kTopThreads) {
        s += __builtin_amdgcn_exp2f((load1<KIND>(xr, i) - m) * a.c);
    }
    s = wave_sum(s);
    __syncthreads();
    if (lane_id() == 0) sh.wave_s[threadIdx.x / kWave] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < kTopWaves; ++w) s += sh.wave_s[w];
    return s;
}

// Appends value(e) to a list in LDS for every e < E that takes(e), with room for `most`; places beyond that are counted, and nothing is written there.
// One addition to the count for the wavefront: each costs the way to LDS and back.
template <int E, class Takes, class Value, class T>
__device__ __forceinline__ void append(T *list, int *count, int most, const Takes &takes, const Value &value)
{
    uint64_t who[E];
    int all = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        who[e] = __ballot(takes(e));
        all += __popcll(who[e]);
    }
    if (all == 0) return;
    int at = 0;
    if (lane_id() == __ffsll((unsigned long long)__ballot(1)) - 1) at = atomicAdd(count, all);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int to = at + __builtin_amdgcn_mbcnt_hi((unsigned)(who[e] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who[e], 0));
        if (takes(e) && to < most) list[to] = value(e);
        at += __popcll(who[e]);
    }
}

// The k largest of the entries found[0 .. n - 1] in sorted, descending, by counting for each how many are larger.
template <int THREADS>
__device__ __forceinline__ void sort_found(const uint64_t *found, int n, int k, uint64_t *sorted)
{
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t own = found[i];
        int rank = 0, j = 0;
#pragma unroll 1
        for (; j + 8 <= n; j += 8)   // eight reads in flight
#pragma unroll
            for (int e = 0; e < 8; ++e) rank += found[j + e] > own;
#pragma unroll 1
        for (; j < n; ++j) rank += found[j] > own;
        if (rank < k) sorted[rank] = own;
    }
}

// The first entries in order of ids whose value is exactly x, behind the `have` in sh.found until there are k.  By one wavefront.
template <int KIND>
__device__ __forceinline__ int take_equal(const void *xr, int begin, int whole, int end, float x, int have, int k, TopShared &sh)
{
    typedef Vec<KIND> V;
    const uint64_t before = ((uint64_t)1 << lane_id()) - 1;
#pragma unroll 1
    for (int base = 0; base <= whole && have < k; base += kWave) {
        const int at = base + lane_id(), i = begin + at * V::kLen;
        const int left = at < whole ? V::kLen : at == whole ? end - i : 0;   // the vector that is not whole is the last
        uint32_t equal = 0;
        for (int e = 0; e < left; ++e) equal |= (uint32_t)(load1<KIND>(xr, i + e) == x) << e;
        int rank = have, all = 0;
        for (int e = 0; e < V::kLen; ++e) {
            const uint64_t who = __ballot(equal >> e & 1);
            rank += __popcll(who & before);
            all += __popcll(who);
        }
        for (int e = 0; e < left; ++e)
            if (equal >> e & 1) {
                if (rank < k) sh.found[rank] = entry_of(order_key(x), (uint32_t)(i + e));
                ++rank;
            }
        have += all;
    }
    return min(have, k);
}

// The top entries of a row with their log probabilities; of a row over kept slots with their target ids.
template <int KIND>
__device__ __forceinline__ void write_top(const TokenArgs &t, int32_t *ids, float *values, int k, int64_t row, const uint64_t *sorted, int n, RowSum r)
{
    if ((int)threadIdx.x < k) {
        const bool in = (int)threadIdx.x < n;
        const uint64_t e = in ? sorted[threadIdx.x] : 0;
        const int32_t at = in ? (int32_t)entry_id(e) : -1;
        ids[row * k + threadIdx.x] = in && t.kept_ids ? t.kept_ids[at] : at;
        values[row * k + threadIdx.x] = in ? log_share<KIND>(key_value(entry_key(e)), r.m, log1pf(r.rest), t.from_most) : -INFINITY;
    }
}

template <int KIND>
__device__ __forceinline__ void write_row(int32_t *ids, float *values, float *lse, int k, float inv_t, int64_t row, const uint64_t *sorted, int n,
                                          SoftStat st)
{
    if ((int)threadIdx.x < k) {
        const bool in = (int)threadIdx.x < n;
        const uint64_t e = in ? sorted[threadIdx.x] : 0;
        ids[row * k + threadIdx.x] = in ? (int32_t)entry_id(e) : -1;
        values[row * k + threadIdx.x] = in ? key_value(entry_key(e)) : KIND == RDK_PROB_F32 ? 0.f : -INFINITY;
    }
    if (lse && threadIdx.x == 0)
        lse[row] = KIND == RDK_PROB_F32 ? logf(st.s) : st.s == 0.f ? -INFINITY : weight_reference(st.m) * inv_t + logf(st.s);
}

// One pass over a part of a row.  Every lane keeps the largest value of its own; if each of the four wavefronts has k / 4 lanes whose largest reaches
// a bound of its own, the least of the four bounds is reached by k of the part's values, and few more exceed it: it is a lower bound of the k-th
// largest.  It is found after the first round of loads and anew as the values seen grow by half (a wavefront reads what the others last
// wrote: bounds only rise, so an old one is a bound too, and nothing waits); a vector whose largest value reaches it is noted by its place.
// What was noted is read again at the end (out of the cache), sifted by the last bound, and sorted.  Where more was noted than there is room for
// (values that rise along the row) the whole part is sifted; where more reaches the last bound than there is room for, by the bound to its last
// bit; and where that is still more, it is the k-th largest value itself and met by many (what masks leave): those above it are
// taken, and the first of those that equal it.
// Only values that crowd in few lanes, and NaN, are left to the search by halving.
// Bound by HBM where rows are many and long: 1024 rows of 151936 fp32 logits, 64 kept, 100 us = 6.2 TB/s, weights 101 us, bf16 58 us = 5.4 TB/s (twice
// the exponentials a byte; without the noting and the end 50 us).  Few rows are a chain: 8 rows of 128256 bf16 logits in 32 parts each
// take 6.7 us, 2.5 of it until the loads are there and the bound stands, 1.3 for sifting, 0.7 for sorting, 0.5 for statistics and stores.
// TOKENS: the sums are those of TokenPass, which also counts the ranks of the row's tokens.
template <int KIND, bool TOKENS>
__global__ __launch_bounds__(kTopThreads) void topk_part_kernel(TopArgs a, std::conditional_t<TOKENS, TokenArgs, NoTokens> t)
{
    static_assert(kRoundVecs == kTokenRoundVecs, "one pass for both");
    typedef Vec<KIND> V;
    constexpr int kRound = kTopThreads * kRoundVecs;    // vectors
    __shared__ TopShared sh;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * a.part_len, end = max(begin, min(a.N, begin + a.part_len));
    const int tid = threadIdx.x, wid = tid / kWave;
    if (a.finished && a.finished[row]) return;
    if (a.scores && a.scores[row] == -INFINITY) return;
    const void *xr = row_ptr<KIND>(a.x, a.ldx, row);
    const char *from = (const char *)xr + (int64_t)begin * V::kSize;
    const int whole = (end - begin) / V::kLen, behind = (end - begin) % V::kLen;   // whole vectors; a value behind them is one thread's each
    // wavefronts that have values, and how many lanes of each have to reach its bound.  The last one is left out where it has fewer lanes with values: it would
    // find no bound, and every value would be wanted (4 rows of 1600 bf16 logits, 128 kept 79 us, 11 without it).
    const int most = min((max(whole, 1) + kWave - 1) / kWave, kTopWaves), lanes = whole - (most - 1) * kWave;
    const int waves = most > 1 && lanes < (a.k + most - 1) / most ? most - 1 : most, share = (a.k + waves - 1) / waves;
    constexpr float none = KIND == RDK_PROB_F32 ? 0.f : -INFINITY;
    float m = none, s = 0.f, ref = 0.f, high = -INFINITY;   // ref: reference of the lane's exponents, times c; high: where it is replaced
    float last = none;
    // Exponents are relative to a value that the lane has seen, not the largest: it is replaced only when a vector exceeds it by 2^60, so the
    // maximum is nothing that the exponentials wait for.  References are rounded products of a value and c, and kept within +-limit,
    // where the rounding is below 1 (at 1e10 it is hundreds, and its exponential no number); rows whose maximum lies outside are summed anew.
    auto raise = [&](float x) __attribute__((always_inline)) {
        const float held = fminf(fmaxf(x, -a.limit), a.limit), to = held * a.c;
        s = s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f(ref - to);
        ref = to;
        high = held + a.margin;
    };
    auto publish = [&](auto bits) __attribute__((always_inline)) {
        const float b = wid < waves ? wave_bound<KIND, decltype(bits)::value>(m, share) : INFINITY;
        if (lane_id() == 0) __hip_atomic_store(&sh.bound[wid], b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    };
    auto least_bound = [&]() __attribute__((always_inline)) {
        float b = INFINITY;
#pragma unroll
        for (int w = 0; w < kTopWaves; ++w) b = fminf(b, __hip_atomic_load(&sh.bound[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        return b;
    };
    if (tid == 0) sh.count = 0;
    [[maybe_unused]] TokenPass<KIND, kTopThreads, true> pass;
    [[maybe_unused]] RowSum row_sum{none, 0.f, 0.f};
    auto begin_tokens = [&]() __attribute__((always_inline)) {
        if constexpr (TOKENS) {
            pass.begin(t, row, xr, begin, begin + whole * V::kLen, a.N);
            if (tid < behind) last = load1<KIND>(from, whole * V::kLen + tid);
            if (behind > 0 && wid == 0) pass.single(t, last, begin + whole * V::kLen + tid);
            m = pass.s.m;
        }
    };
    if (!TOKENS && tid < behind) {
        last = load1<KIND>(from, whole * V::kLen + tid);
        m = fmaxf(m, last);
        if (KIND == RDK_PROB_F32) {
            s = last;
        } else {
            if (last > high) raise(last);
            s = __builtin_amdgcn_exp2f(fmaf(last, a.c, -ref));
        }
    }
    float tau = INFINITY;
    int next_bound = 0, round = 0, noted = 0;
    // Always as many loads, of the last vector where the round has none of its own: the compiler counts loads in flight, and would wait for all of
    // them behind a branch that has some of its own (1024 rows of 151936 bf16 logits 61 us).
    auto load_round = [&](u32x4 (&raw)[kRoundVecs], int base, auto first) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) {
            const u32x4_any *at = (const u32x4_any *)(from + (uint64_t)(uint32_t)min(base + j * kTopThreads + tid, whole - 1) * 16);
            raw[j] = decltype(first)::value ? *at : __builtin_nontemporal_load(at);   // a part of one round is read again at once
        }
    };
    auto take_round = [&](u32x4 (&now)[kRoundVecs], int base) __attribute__((always_inline)) {
        if (base + kRound > whole) {
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j)
                if (base + j * kTopThreads + tid >= whole) now[j] = V::fill();
        }
        float vm[kRoundVecs];
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) {
            if constexpr (TOKENS) {
                vm[j] = pass.vector(t, now[j]);
                continue;
            }
            float v[V::kLen], sum = 0.f;
            V::to(now[j], v);
            vm[j] = V::largest(v, none);
            if constexpr (KIND == RDK_PROB_F32) {
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) sum += v[e];
            } else {
                if (vm[j] > high) raise(vm[j]);
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) sum += __builtin_amdgcn_exp2f(fmaf(v[e], a.c, -ref));
            }
            s += sum;
        }
        m = max3(m, max3(vm[0], vm[1], vm[2]), vm[3]);
        if constexpr (TOKENS)
            if (t.rank) pass.ranks(t, now, max3(max3(vm[0], vm[1], vm[2]), vm[3], none), base);
        if (round == next_bound) {
            next_bound = round + 1 + round / 2;
            publish(std::integral_constant<int, 16>());
            if (round == 0) __syncthreads();
            tau = least_bound();
        }
        ++round;
        // every wavefront notes in a list of its own, whose length it alone knows
        uint64_t who[kRoundVecs], any = 0;
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) any |= who[j] = __ballot(vm[j] >= tau);
        if (any) {
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j) {
                const int to = noted + __builtin_amdgcn_mbcnt_hi((unsigned)(who[j] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who[j], 0));
                if (vm[j] >= tau && to < kNoted) sh.queue[wid][to] = make_float2(vm[j], __int_as_float(base + j * kTopThreads + tid));
                noted += __popcll(who[j]);
            }
        }
    };
    static_assert(kRoundVecs == 4 && kTopWaves == 4, "the largest of a round is formed of four");
    if (whole > 0) {
        u32x4 raw[kRoundVecs], ahead[kRoundVecs];   // in turn: the round at hand, and the next one on its way
        load_round(raw, 0, std::true_type());
        begin_tokens();
#pragma unroll 1
        for (int base = 0;; base += 2 * kRound) {
            load_round(ahead, base + kRound, std::false_type());
            take_round(raw, base);
            if (base + kRound >= whole) break;
            load_round(raw, base + 2 * kRound, std::false_type());
            take_round(ahead, base + kRound);
            if (base + 2 * kRound >= whole) break;
        }
    }
    if (whole == 0) begin_tokens();
    // statistics of the part, and its last bound
    if constexpr (TOKENS) {
        pass.s.m = m;
        row_sum = pass.finish(t, from, whole, behind, token_shared<TOKENS>());
    }
    const float wave_m = wave_max(m);
    if constexpr (!TOKENS && KIND != RDK_PROB_F32) {
        const float to = fminf(fmaxf(wave_m, -a.limit), a.limit) * a.c;
        s = s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f(ref - to);
    }
    const float wave_s = wave_sum(s);
    if (lane_id() == 0) {
        sh.wave_m[wid] = wave_m;
        sh.wave_s[wid] = wave_s;
        sh.noted[wid] = noted;
    }
    if (round != 1) publish(std::integral_constant<int, 16>());
    __syncthreads();
    tau = least_bound();
    SoftStat stat{none, 0.f};
#pragma unroll
    for (int w = 0; w < kTopWaves; ++w) stat.m = fmaxf(stat.m, sh.wave_m[w]);
    if constexpr (TOKENS) {
        stat.s = row_sum.rest;   // (looked at for NaN)
    } else if constexpr (KIND == RDK_PROB_F32) {
#pragma unroll
        for (int w = 0; w < kTopWaves; ++w) stat.s += sh.wave_s[w];
    } else {
        const float held = fminf(fmaxf(stat.m, -a.limit), a.limit), to = held * a.c;
#pragma unroll
        for (int w = 0; w < kTopWaves; ++w) {
            const float by = fminf(fmaxf(sh.wave_m[w], -a.limit), a.limit) * a.c;
            stat.s += sh.wave_s[w] == 0.f ? 0.f : sh.wave_s[w] * __builtin_amdgcn_exp2f(by - to);
        }
        stat.s *= __builtin_amdgcn_exp2f(-fmaf(held, a.c, -to));   // the rounding of the reference itself
        if (stat.m > -INFINITY && fabsf(stat.m) > a.limit) stat.s = wide_sum<KIND>(a, xr, begin, end, stat.m, sh);
    }
    const bool nan = stat.s != stat.s;
    bool all = max(max(sh.noted[0], sh.noted[1]), max(sh.noted[2], sh.noted[3])) > kNoted;   // the whole part is sifted
    int n = 0, stage = 0;   // 0: what reaches the bound; 1: the bound to the last bit; 2: what exceeds it
    float least = tau;
#pragma unroll 1
    while (!nan) {
        const int count = all ? whole : noted, stride = all ? kTopThreads : kWave, own = all ? tid : lane_id();
#pragma unroll 1
        for (int first = 0; first < count; first += kSift * stride) {   // (alike for the wavefront, for which append() speaks)
            u32x4 raw[kSift];
            int at[kSift];
#pragma unroll
            for (int j = 0; j < kSift; ++j) {   // together on their way
                const int q = first + j * stride + own;
                const float2 seen = !all && q < count ? sh.queue[wid][q] : make_float2(INFINITY, __int_as_float(q));
                at[j] = q < count && seen.x >= least ? __float_as_int(seen.y) : -1;
                raw[j] = V::fill();
                if (at[j] >= 0) raw[j] = *(const u32x4_any *)(from + (int64_t)at[j] * 16);
            }
#pragma unroll 1
            for (int j = 0; j < kSift && first + j * stride < count; ++j) {
                float v[V::kLen];
                V::to(raw[0], v);
                append<V::kLen>(
                    sh.found, &sh.count, kFound, [&](int e) { return v[e] >= least; },
                    [&](int e) { return entry_of(order_key(v[e]), (uint32_t)(begin + at[0] * V::kLen + e)); });
#pragma unroll
                for (int i = 0; i + 1 < kSift; ++i) raw[i] = raw[i + 1], at[i] = at[i + 1];
            }
        }
        if (tid < behind)
            append<1>(
                sh.found, &sh.count, kFound, [&](int) { return last >= least; },
                [&](int) { return entry_of(order_key(last), (uint32_t)(begin + whole * V::kLen + tid)); });
        __syncthreads();
        n = sh.count;
        if (n <= kFound || stage == 2) break;
        all = true;
        stage = KIND == RDK_LOGIT_BF16 ? 2 : stage + 1;
        if (stage == 1) publish(std::integral_constant<int, 32>());
        __syncthreads();
        if (tid == 0) sh.count = 0;
        tau = least_bound();
        least = stage == 2 ? key_value(order_key(tau) + 1) : tau;
        __syncthreads();
    }
    if (stage == 2 && n < a.k) {
        __syncthreads();
        if (wid == 0) {
            const int filled = take_equal<KIND>(xr, begin, whole, end, tau, n, a.k, sh);
            if (tid == 0) sh.count = filled;
        }
        __syncthreads();
        n = sh.count;
    }
    if (nan || n > kFound) {
        const uint32_t masked = masked_key<KIND>();
        n = select_exact<kTopThreads>(
            [&](auto f) {
                for (int i = begin + tid; i < end; i += kTopThreads) {
                    const uint32_t key = order_key(load1<KIND>(xr, i));
                    f(key > masked ? entry_of(key, (uint32_t)i) : (uint64_t)0);
                }
            },
            a.k, sh.slow);
    } else {
        sort_found<kTopThreads>(sh.found, n, a.k, sh.slow.sorted);
        n = min(n, a.k);
        __syncthreads();
    }
    if (a.entries) {
        // the best of every part and beam first, then the second best of every one, ...
        const uint32_t group = (uint32_t)row / (uint32_t)a.W, beam = (uint32_t)row % (uint32_t)a.W;
        if (tid < a.k) a.entries[(((int64_t)group * a.k + tid) * a.parts + part) * a.W + beam] = tid < n ? sh.slow.sorted[tid] : 0;
        if constexpr (TOKENS) {
            if (wid == 0) pass.write_part(t, row, part, a.parts, row_sum, token_shared<TOKENS>());
        } else if (tid == 0) {
            a.stat[row * a.parts + part] = stat;
        }
        return;
    }
    if constexpr (TOKENS) {
        if (wid == 0) write_tokens<KIND>(t, row, row_sum, pass.place, pass.value, pass.counted(t, token_shared<TOKENS>()));
        write_top<KIND>(t, a.ids, a.values, a.k, row, sh.slow.sorted, n, row_sum);
        return;
    }
    write_row<KIND>(a.ids, a.values, a.lse, a.k, a.inv_t, row, sh.slow.sorted, n, stat);
}

// A lane's first partial statistics of a row.
template <int KIND>
__device__ __forceinline__ SoftStat first_stat(const SoftStat *stat, int parts)
{
    return lane_id() < parts ? stat[lane_id()] : SoftStat{KIND == RDK_PROB_F32 ? 0.f : -INFINITY, 0.f};
}

// Partial statistics of a row brought together, by a wavefront that has read the first.
template <int KIND>
__device__ __forceinline__ SoftStat merge_stats(SoftStat first, const SoftStat *stat, int parts, float c)
{
    SoftStat r = first;
    for (int p = lane_id() + kWave; p < parts; p += kWave) {
        const SoftStat o = stat[p];
        if (KIND == RDK_PROB_F32) {
            r.m = fmaxf(r.m, o.m);
            r.s += o.s;
        } else {
            const float m = fmaxf(r.m, o.m), ref = weight_reference(m);
            r.s = (r.s == 0.f ? 0.f : r.s * __builtin_amdgcn_exp2f((weight_reference(r.m) - ref) * c)) +
                  (o.s == 0.f ? 0.f : o.s * __builtin_amdgcn_exp2f((weight_reference(o.m) - ref) * c));
            r.m = m;
        }
    }
    const float m = wave_max(r.m);
    if (KIND != RDK_PROB_F32) r.s = r.s == 0.f ? 0.f : r.s * __builtin_amdgcn_exp2f((weight_reference(r.m) - weight_reference(m)) * c);
    return SoftStat{m, wave_sum(r.s)};
}

template <int THREADS>
struct MergeShared {
    SelectShared slow;
    uint64_t found[kFound];
    uint32_t keys[THREADS];
    int count;
};

// The k largest of the workgroup's `count` entries in sh.slow.sorted; returns how many there are.  Thread t holds the entries t, t + THREADS, ... in
// own (0: none).  By a bound as above: the entries come best places first, so no entry of a thread is much larger than its first.  The
// largest of four wavefronts are looked at together; sixteen find a bound each, of which the least is taken (beams stand next to one
// another: every wavefront has its share of the best ones).
template <int THREADS, int EACH, int BITS>
__device__ __forceinline__ int select_entries(const uint64_t (&own)[EACH], int count, int k, MergeShared<THREADS> &sh)
{
    constexpr int kWaves = THREADS / kWave;
    const int tid = threadIdx.x;
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) best = own[i] > best ? own[i] : best;
    if (tid == 0) sh.count = 0;
    uint32_t bound = 0;
    if constexpr (kWaves <= 4) {
        sh.keys[tid] = entry_key(best);
        __syncthreads();
        uint32_t keys[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) keys[w] = sh.keys[w * kWave + lane_id()];
#pragma unroll 4
        for (int bit = 31; bit >= 32 - BITS; --bit) {
            const uint32_t tried = bound | (1u << bit);
            int n = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) n += __popcll(__ballot(keys[w] >= tried));
            if (n >= k) bound = tried;
        }
    } else {
        const int waves = min((count + kWave - 1) / kWave, kWaves);
        const uint32_t b = tid / kWave < waves ? wave_nth<BITS>(entry_key(best), (k + waves - 1) / waves) : 0xFFFFFFFFu;
        if (lane_id() == 0) sh.keys[tid / kWave] = b;
        __syncthreads();
        bound = sh.keys[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) bound = min(bound, sh.keys[w]);
    }
    const uint64_t least = bound ? (uint64_t)bound << 32 : 1;
    append<EACH>(
        sh.found, &sh.count, kFound, [&](int i) { return own[i] >= least; }, [&](int i) { return own[i]; });
    __syncthreads();
    const int n = sh.count;
    if (n > kFound)   // thousands that tie with the k-th, or beams of which few have all the best
        return select_exact<THREADS>(
            [&](auto f) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) f(own[i]);
            },
            k, sh.slow);
    sort_found<THREADS>(sh.found, n, k, sh.slow.sorted);
    __syncthreads();
    return min(n, k);
}

struct TopMergeArgs {
    const void *x;        // TOKENS: the rows
    int64_t ldx;
    const uint64_t *entries;
    const SoftStat *stat;
    int k, parts;
    float inv_t, c;
    int32_t *ids;
    float *values, *lse;
};

// The parts of a row brought together.  A chain of reads of the caches, a search of a step a bit and a sort: 4.0 us with its launch for 8 rows of 32
// parts and 16 kept (512 entries a row; bf16 keys have 16 bits that matter, others are searched to 24: with 32 4.5 us).
template <int KIND, int EACH, bool TOKENS>
__global__ __launch_bounds__(kTopThreads) void topk_merge_kernel(TopMergeArgs a, std::conditional_t<TOKENS, TokenArgs, NoTokens> t)
{
    __shared__ MergeShared<kTopThreads> sh;
    const int64_t row = blockIdx.x;
    const int count = a.parts * a.k;
    uint64_t own[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = i * kTopThreads + (int)threadIdx.x;
        own[i] = at < count ? a.entries[row * count + at] : 0;
    }
    if constexpr (TOKENS) {
        __shared__ RowSum row_sum;
        if (threadIdx.x < kWave) {
            const RowSum r = merge_tokens<KIND>(t, row, row_ptr<KIND>(a.x, a.ldx, row), a.parts);
            if (threadIdx.x == 0) row_sum = r;
        }
        const int n = select_entries<kTopThreads, EACH, KIND == RDK_LOGIT_BF16 ? 16 : 24>(own, count, a.k, sh);
        write_top<KIND>(t, a.ids, a.values, a.k, row, sh.slow.sorted, n, row_sum);
        return;
    }
    SoftStat stat{0.f, 0.f};
    if (threadIdx.x < kWave) stat = merge_stats<KIND>(first_stat<KIND>(a.stat + row * a.parts, a.parts), a.stat + row * a.parts, a.parts, a.c);
    const int n = select_entries<kTopThreads, EACH, KIND == RDK_LOGIT_BF16 ? 16 : 24>(own, count, a.k, sh);
    write_row<KIND>(a.ids, a.values, a.lse, a.k, a.inv_t, row, sh.slow.sorted, n, stat);
}

struct BeamArgs {
    const uint64_t *entries;
    const SoftStat *stat;
    const float *scores;
    const uint8_t *finished;
    int W, N, k, K, parts, eos;
    float *scores_out;
    int32_t *parent, *token;
    uint8_t *finished_out;
};

// One request: scores of its beams' candidates, and the K best of them.  The same chain and the beams' logarithms: 5.2 us for a request of 4 beams
// of 128256 ids, 4 kept (512 entries), 5.7 us for 16 requests of 8 beams, 8 kept (6.2 with their statistics asked for one after the other).
template <int KIND, int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void beam_merge_kernel(BeamArgs a)
{
    __shared__ MergeShared<THREADS> sh;
    __shared__ float beam_m[kWave], beam_log[kWave], beam_score[kWave];
    __shared__ int beam_state[kWave];        // 0: no candidates, 1: finished, 2: live
    const int64_t g = blockIdx.x, b0 = g * a.W;
    const int tid = threadIdx.x, lists = a.W * a.parts, count = lists * a.k;
    const float per_beam = 1.f / a.W;
    uint64_t own[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {         // (of beams without a row this is whatever lay there, and not used)
        const int at = i * THREADS + tid;
        own[i] = at < count ? a.entries[g * count + at] : 0;
    }
    constexpr int kWaves = THREADS / kWave, kAhead = 4;
    const float scores = lane_id() < a.W ? a.scores[b0 + lane_id()] : -INFINITY;   // a beam to a lane
    const int over = a.finished && lane_id() < a.W ? a.finished[b0 + lane_id()] : 0;
#pragma unroll 1
    for (int first = tid / kWave; first < a.W; first += kAhead * kWaves) {
        SoftStat ahead[kAhead];   // (of beams without a row whatever lay there, and not used)
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ahead[j] = first_stat<KIND>(a.stat + (b0 + min(first + j * kWaves, a.W - 1)) * a.parts, a.parts);
#pragma unroll 1
        for (int j = 0; j < kAhead && first + j * kWaves < a.W; ++j) {
            const int w = first + j * kWaves;
            const float score = __shfl(scores, w);
            const int state = score == -INFINITY ? 0 : __shfl(over, w) ? 1 : 2;
            SoftStat st = merge_stats<KIND>(ahead[0], a.stat + (b0 + w) * a.parts, a.parts, kLog2e);
            if (state != 2) st = SoftStat{0.f, 0.f};
            if (lane_id() == 0) {
                beam_score[w] = score;
                beam_state[w] = state;
                beam_m[w] = weight_reference(st.m);
                beam_log[w] = KIND == RDK_PROB_F32 ? st.s : logf(st.s);
            }
#pragma unroll
            for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int at = i * THREADS + tid;
        const int w = at - (int)(((float)at + 0.5f) * per_beam) * a.W;   // at % W (numbers below 2^15: exact)
        const int state = at < count ? beam_state[w] : 0;
        uint64_t e = own[i];
        if (state == 1) {
            e = at < a.W ? entry_of(order_key(beam_score[w]), (uint32_t)w * a.N + a.eos) : 0;
        } else if (state == 2 && e != 0) {
            const float x = key_value(entry_key(e));
            const float score = beam_score[w] + (KIND == RDK_PROB_F32 ? logf(x / beam_log[w]) : (x - beam_m[w]) - beam_log[w]);
            e = score == -INFINITY ? 0 : entry_of(order_key(score), (uint32_t)w * a.N + entry_id(e));
        } else {
            e = 0;
        }
        own[i] = e;
    }
    const int n = select_entries<THREADS, EACH, 24>(own, count, a.K, sh);
    if (tid < a.K) {
        const bool in = tid < n;
        const uint64_t e = in ? sh.slow.sorted[tid] : 0;
        const int w = in ? (int)(entry_id(e) / (uint32_t)a.N) : -1, j = in ? (int)(entry_id(e) % (uint32_t)a.N) : -1;
        const int64_t o = g * a.K + tid;
        a.scores_out[o] = in ? key_value(entry_key(e)) : -INFINITY;
        a.parent[o] = w;
        a.token[o] = j;
        if (a.finished_out) a.finished_out[o] = in && (j == a.eos || beam_state[w] == 1);
    }
}

template <class F>
void with_kind(rdk_input_kind_t kind, const F &f)
{
    if (kind == RDK_PROB_F32) f(std::integral_constant<int, RDK_PROB_F32>());
    else if (kind == RDK_LOGIT_F32) f(std::integral_constant<int, RDK_LOGIT_F32>());
    else f(std::integral_constant<int, RDK_LOGIT_BF16>());
}

// How a row is read in parts, so that a batch of few rows fills the chip: two workgroups to a compute unit, parts of whole rounds of loads or at least
// 4096 values (16 requests of 8 beams over 128256 bf16 ids: 256, 512, 1024, 2048 workgroups 22.1, 21.0, 22.3, 22.5 us; 64 of 4 26.7, 24.0, 27.0,
// 29.8).  Where the merge of the parts is a launch that a whole row does without (topk), rows of up to six rounds and batches of 192 rows and
// more are not split: in one part and in two to four 192 rows of 32000 bf16 logits take 11.0 and 13.3 us, 128 rows 10.5 and 12.6, 192 of
// 128256 23.9 and 25.9; but 128 rows of 128256 21.2 and 19.5.
struct Parts {
    int count, len;
};
Parts parts_of(int64_t rows, int N, rdk_input_kind_t kind, int most, bool merges)
{
    const int round = kTopThreads * kRoundVecs * (kind == RDK_LOGIT_BF16 ? 8 : 4);
    const int want = !merges && (rows >= 192 || N <= 6 * round) ? 1 : (int)(512 / rows);
    if (want <= 1 || N <= 4096 || most <= 1) return Parts{1, (int)align_up(N, 64)};
    int64_t len = ((int64_t)N - 1) / (want < most ? want : most) + 1;
    if (len < 4096) len = 4096;
    if (len > round && want <= most) len = len / round * round;
    len = (int64_t)align_up((size_t)len, 64);
    int count = (int)((N - 1) / len) + 1;
    if (count > most) {
        len = (int64_t)align_up((size_t)((N - 1) / most + 1), 64);
        count = (int)((N - 1) / len) + 1;
    }
    return Parts{count, (int)len};
}

struct TopWs {
    uint64_t *entries;
    SoftStat *stat;
};

TopWs carve(int64_t rows, int parts, int k, void *ws, size_t *bytes)
{
    TopWs w;
    char *p = (char *)ws;
    w.entries = (uint64_t *)p; p += align_up((size_t)rows * parts * k * sizeof(uint64_t), 256);
    w.stat = (SoftStat *)p; p += align_up((size_t)rows * parts * sizeof(SoftStat), 256);
    if (bytes) *bytes = (size_t)(p - (char *)ws);
    return w;
}

TopArgs part_args(RowInput x, int N, int k, Parts parts, float temperature)
{
    TopArgs a{};
    a.x = x.ptr; a.ldx = x.ld; a.N = N; a.k = k; a.parts = parts.count; a.part_len = parts.len; a.W = 1;
    a.inv_t = 1.f / temperature;
    a.c = a.inv_t * kLog2e;
    a.margin = 60.f / a.c;
    // 2^24 / c: the product of a value and c is rounded by 1/2 at most, and exp2 of that is no more than a factor of the sums.  (2^100 at most: c may be tiny.)
    a.limit = a.c > 0x1p-76f ? 0x1p24f / a.c : 0x1p100f;
    return a;
}

}  // namespace

int select_max_entries() { return kMaxTop; }
int select_max_ids() { return 1 << 30; }   // places in a row, a round of loads behind its end among them, are 32-bit numbers

static Parts topk_parts(const rdk_topk_desc_t &d, rdk_input_kind_t kind) { return parts_of(d.B, d.N, kind, kMergeEntries / d.k, false); }

size_t topk_workspace_bytes(const rdk_topk_desc_t &d, rdk_input_kind_t kind)
{
    const int parts = topk_parts(d, kind).count;
    size_t bytes = 0;
    if (parts > 1) carve(d.B, parts, d.k, nullptr, &bytes);
    return bytes;
}

rdk_status_t launch_topk(const rdk_topk_desc_t &d, RowInput x, int32_t *ids, float *values, float *lse, void *ws, hipStream_t st)
{
    const Parts split = topk_parts(d, x.kind);
    const int parts = split.count;
    TopArgs a = part_args(x, d.N, d.k, split, d.temperature);
    a.ids = ids; a.values = values; a.lse = lse;
    if (parts > 1) {
        const TopWs w = carve(d.B, parts, d.k, ws, nullptr);
        a.entries = w.entries;
        a.stat = w.stat;
    }
    with_kind(x.kind, [&](auto kind) {
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<decltype(kind)::value, false>), dim3((unsigned)d.B * parts), dim3(kTopThreads), 0, st, a,
                         NoTokens{});
        if (parts > 1) {
            constexpr int KIND = decltype(kind)::value;
            const TopMergeArgs m{nullptr, 0, a.entries, a.stat, d.k, parts, a.inv_t, a.c, ids, values, lse};
            if (parts * d.k <= 4 * kTopThreads)
                RDK_TIMED_LAUNCH("topk_merge_kernel", (topk_merge_kernel<KIND, 4, false>), dim3((unsigned)d.B), dim3(kTopThreads), 0, st, m, NoTokens{});
            else
                RDK_TIMED_LAUNCH("topk_merge_kernel", (topk_merge_kernel<KIND, 16, false>), dim3((unsigned)d.B), dim3(kTopThreads), 0, st, m, NoTokens{});
        }
    });
    RDK_LAUNCH_CHECK("topk_part_kernel");
    return RDK_OK;
}

static Parts logprobs_top_parts(const rdk_logprobs_desc_t &d, rdk_input_kind_t kind)
{
    const int most = kMergeEntries / d.k;
    return parts_of(d.B, d.N, kind, most < kWave ? most : kWave, false);   // (the tokens' merge has a lane to a part)
}

static size_t carve_tokens(const rdk_logprobs_desc_t &d, int parts, TokenArgs &t, TopWs &w, void *ws)
{
    size_t bytes = 0;
    w = carve(d.B, parts, d.k, ws, &bytes);
    return bytes + token_places(t, (char *)ws + bytes, d.B, parts);
}

size_t logprobs_top_workspace_bytes(const rdk_logprobs_desc_t &d, rdk_input_kind_t kind)
{
    const int parts = logprobs_top_parts(d, kind).count;
    TokenArgs t{};
    TopWs w;
    t.C = d.C;
    return parts > 1 ? carve_tokens(d, parts, t, w, nullptr) : 0;
}

rdk_status_t launch_logprobs_top(const rdk_logprobs_desc_t &d, RowInput x, TokenArgs t, int32_t *top_ids, float *top_logprobs, void *ws, hipStream_t st)
{
    const Parts split = logprobs_top_parts(d, x.kind);
    const int parts = split.count;
    TopArgs a = part_args(x, d.N, d.k, split, d.temperature);
    a.ids = top_ids; a.values = top_logprobs;
    TopWs w{};
    if (parts > 1) {
        carve_tokens(d, parts, t, w, ws);
        a.entries = w.entries;
    }
    with_kind(x.kind, [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<KIND, true>), dim3((unsigned)d.B * parts), dim3(kTopThreads),
                         before_tokens_bytes(t, kTopThreads), st, a, t);
        if (parts > 1) {
            const TopMergeArgs m{x.ptr, x.ld, a.entries, nullptr, d.k, parts, a.inv_t, a.c, top_ids, top_logprobs, nullptr};
            if (parts * d.k <= 4 * kTopThreads)
                RDK_TIMED_LAUNCH("topk_merge_kernel", (topk_merge_kernel<KIND, 4, true>), dim3((unsigned)d.B), dim3(kTopThreads), 0, st, m, t);
            else
                RDK_TIMED_LAUNCH("topk_merge_kernel", (topk_merge_kernel<KIND, 16, true>), dim3((unsigned)d.B), dim3(kTopThreads), 0, st, m, t);
        }
    });
    RDK_LAUNCH_CHECK("topk_part_kernel");
    return RDK_OK;
}

static Parts beam_parts(const rdk_beam_desc_t &d, rdk_input_kind_t kind, int k) { return parts_of((int64_t)d.G * d.W, d.N, kind, kBeamEntries / (d.W * k), true); }

size_t beam_select_workspace_bytes(const rdk_beam_desc_t &d, rdk_input_kind_t kind)
{
    const int k = d.K < d.N ? d.K : d.N;
    size_t bytes = 0;
    carve((int64_t)d.G * d.W, beam_parts(d, kind, k).count, k, nullptr, &bytes);
    return bytes;
}

rdk_status_t launch_beam_select(const rdk_beam_desc_t &d, RowInput x, const float *scores, const uint8_t *finished, float *scores_out,
                                int32_t *parent, int32_t *token, uint8_t *finished_out, void *ws, hipStream_t st)
{
    const int k = d.K < d.N ? d.K : d.N;
    const Parts split = beam_parts(d, x.kind, k);
    const int parts = split.count;
    const TopWs w = carve((int64_t)d.G * d.W, parts, k, ws, nullptr);
    TopArgs a = part_args(x, d.N, k, split, 1.f);
    a.scores = scores; a.finished = finished;
    a.entries = w.entries; a.stat = w.stat; a.W = d.W;
    BeamArgs b{};
    b.entries = w.entries; b.stat = w.stat; b.scores = scores; b.finished = finished;
    b.W = d.W; b.N = d.N; b.k = k; b.K = d.K; b.parts = parts; b.eos = d.eos;
    b.scores_out = scores_out; b.parent = parent; b.token = token; b.finished_out = finished_out;
    with_kind(x.kind, [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<KIND, false>), dim3((unsigned)(d.G * d.W) * parts), dim3(kTopThreads), 0, st, a,
                         NoTokens{});
        const int count = d.W * parts * k;
        if (count <= 4 * 256)
            RDK_TIMED_LAUNCH("beam_merge_kernel", (beam_merge_kernel<KIND, 256, 4>), dim3((unsigned)d.G), dim3(256), 0, st, b);
        else if (count <= 16 * 256)
            RDK_TIMED_LAUNCH("beam_merge_kernel", (beam_merge_kernel<KIND, 256, 16>), dim3((unsigned)d.G), dim3(256), 0, st, b);
        else
            RDK_TIMED_LAUNCH("beam_merge_kernel", (beam_merge_kernel<KIND, 1024, 16>), dim3((unsigned)d.G), dim3(1024), 0, st, b);
    });
    RDK_LAUNCH_CHECK("beam_merge_kernel");
    return RDK_OK;
}

}  // namespace rdk
