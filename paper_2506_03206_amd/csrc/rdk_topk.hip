// The k largest entries of rows over a vocabulary with the logarithm of their normaliser, and beam search's selection over beams and
// vocabulary, which takes the K largest entries of every live beam and merges them per request.
#include "rdk_select.hpp"
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kTopThreads = 256;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

constexpr int kRoundVecs = 4;          // 16-byte vectors of a lane in a round
constexpr int kQueue = 1024;           // vectors noted, entries sorted: what exceeds it takes the slow way
constexpr int kMergeEntries = 2048;    // of a row's parts together
constexpr int kBeamEntries = 4096;     // of a request's beams and their parts together

struct TopArgs {
    const void *x;
    int64_t ldx;
    int N, k, parts, part_len;
    float inv_t, c, limit;  // c = log2(e) / temperature; rows with a maximum beyond +-limit take the slow way
    // rows of beams that have no candidates among the ids are passed over
    const float *scores;
    const uint8_t *finished;
    uint64_t *entries;      // [rows, parts, k], 0 where a part has fewer; or NULL: the outputs of topk itself
    SoftStat *stat;         // [rows, parts]
    int32_t *ids;
    float *values, *lse;
};

struct TopShared {
    SelectShared slow;
    uint64_t found[kQueue];
    uint32_t keys[kTopThreads], queue[kQueue];
    float wave_m[kTopThreads / kWave], wave_s[kTopThreads / kWave];
    float tau;
    int queued, count;
};

// A lower bound of the k-th largest of the values whose largest per lane are in sh.keys, to sixteen bits: the k-th largest of those.  By wave 0.
template <int KIND>
__device__ __forceinline__ float bound_of(const uint32_t (&own)[kTopThreads / kWave], int k)
{
    uint32_t found = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t tried = found | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < kTopThreads / kWave; ++i) n += __popcll(__ballot(own[i] >= tried));
        if (n >= k) found = tried;
    }
    const uint32_t key = found << 16;
    // fewer than k lanes have an unmasked value: every unmasked one is wanted
    if (key <= masked_key<KIND>()) return KIND == RDK_PROB_F32 ? __uint_as_float(1u) : -3.402823466e38f;
    return key_value(key);
}

// Statistics of a part (m the largest value, s the sum of exp((x - m) / T)) and its k largest by halving: for rows that the fast way does not hold.
template <int KIND>
__device__ __noinline__ int slow_part(const TopArgs &a, const void *xr, int begin, int end, TopShared &sh, SoftStat *stat)
{
    float m = KIND == RDK_PROB_F32 ? 0.f : -INFINITY, s = 0.f;
    for (int i = begin + (int)threadIdx.x; i < end; i += kTopThreads) m = fmaxf(m, load1<KIND>(xr, i));
    m = wave_max(m);
    __syncthreads();
    if (lane_id() == 0) sh.wave_m[threadIdx.x / kWave] = m;
    __syncthreads();
    for (int w = 0; w < kTopThreads / kWave; ++w) m = fmaxf(m, sh.wave_m[w]);
    const float ref = weight_reference(m);
    for (int i = begin + (int)threadIdx.x; i < end; i += kTopThreads) {
        const float x = load1<KIND>(xr, i);
        s += KIND == RDK_PROB_F32 ? x : __builtin_amdgcn_exp2f((x - ref) * a.c);
    }
    s = wave_sum(s);
    if (lane_id() == 0) sh.wave_s[threadIdx.x / kWave] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < kTopThreads / kWave; ++w) s += sh.wave_s[w];
    *stat = SoftStat{m, s};
    const uint32_t masked = masked_key<KIND>();
    return select_exact<kTopThreads>(
        [&](int64_t i) {
            const uint32_t key = order_key(load1<KIND>(xr, begin + i));
            return key > masked ? entry_of(key, (uint32_t)(begin + i)) : 0;
        },
        end - begin, a.k, sh.slow);
}

__device__ __forceinline__ void note(uint32_t *queue, int *count, uint32_t what)
{
    const int at = atomicAdd(count, 1);
    if (at < kQueue) queue[at] = what;
}

// The k largest of the entries found[0 .. n - 1] in sorted, descending, by counting for each how many are larger.
__device__ __forceinline__ void sort_found(const uint64_t *found, int n, int k, uint64_t *sorted)
{
    for (int i = threadIdx.x; i < n; i += kTopThreads) {
        const uint64_t own = found[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += found[j] > own;
        if (rank < k) sorted[rank] = own;
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

// One pass over a part of a row.  Every lane keeps the largest value of its own; the k-th largest of those 256 is a lower bound of the part's k-th
// largest that only some k of the part's values exceed, so few vectors have to be looked at again.  The bound is found after the first
// round of loads and anew whenever the values seen have doubled; a vector whose largest value reaches it is noted by its place.  What was
// noted is read again at the end (out of the cache), sifted by the final bound, and sorted.
template <int KIND>
__global__ __launch_bounds__(kTopThreads) void topk_part_kernel(TopArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kWaves = kTopThreads / kWave, kRound = kTopThreads * kRoundVecs * V::kLen;
    __shared__ TopShared sh;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * a.part_len, end = min(a.N, begin + a.part_len);
    const int tid = threadIdx.x, wid = tid / kWave;
    if (a.finished && a.finished[row]) return;
    if (a.scores && a.scores[row] == -INFINITY) return;
    const void *xr = row_ptr<KIND>(a.x, a.ldx, row);
    const float none = KIND == RDK_PROB_F32 ? 0.f : -INFINITY;
    float m = none, s = 0.f, ref = 0.f;     // ref: reference of the lane's exponents, times c
    float tau = INFINITY;
    u32x4 raw[kRoundVecs];
    auto load_round = [&](int base) {
        if (base + kRound <= end) {
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j) raw[j] = *(const u32x4_any *)((const char *)xr + (int64_t)(base + (j * kTopThreads + tid) * V::kLen) * V::kSize);
        } else {
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j) {
                const int i = base + (j * kTopThreads + tid) * V::kLen;
                raw[j] = i < end ? V::load(xr, i, end) : V::fill();
            }
        }
    };
    if (tid == 0) sh.queued = sh.count = 0;
    load_round(begin);
    int next_bound = 0, round = 0;
    for (int base = begin; base < end; base += kRound, ++round) {
        u32x4 now[kRoundVecs];
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) now[j] = raw[j];
        if (base + kRound < end) load_round(base + kRound);
        float vm[kRoundVecs];
        float v[V::kLen];
        float mx = m;
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j) {
            V::to(now[j], v);
            vm[j] = v[0];
#pragma unroll
            for (int e = 1; e < V::kLen; ++e) vm[j] = fmaxf(vm[j], v[e]);
            mx = fmaxf(mx, vm[j]);
        }
        if constexpr (KIND == RDK_PROB_F32) {
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j) {
                V::to(now[j], v);
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) s += v[e];
            }
        } else {
            const float to = fminf(fmaxf(mx, -a.limit), a.limit) * a.c;
            s = s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f(ref - to);
            ref = to;
#pragma unroll
            for (int j = 0; j < kRoundVecs; ++j) {
                V::to(now[j], v);
                float part_sum = 0.f;
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) part_sum += __builtin_amdgcn_exp2f(fmaf(v[e], a.c, -to));
                s += part_sum;
            }
        }
        m = mx;
        if (round == next_bound) {      // the same for the whole workgroup
            next_bound = 2 * round + 1;
            sh.keys[tid] = order_key(m) >> 16;
            __syncthreads();
            if (wid == 0) {
                uint32_t own[kWaves];
#pragma unroll
                for (int i = 0; i < kWaves; ++i) own[i] = sh.keys[i * kWave + lane_id()];
                const float bound = bound_of<KIND>(own, a.k);
                if (tid == 0) sh.tau = bound;
            }
            __syncthreads();
            tau = sh.tau;
        }
#pragma unroll
        for (int j = 0; j < kRoundVecs; ++j)
            if (vm[j] >= tau) note(sh.queue, &sh.queued, (uint32_t)(base - begin) / V::kLen + j * kTopThreads + tid);
    }
    // statistics of the part
    const float wave_m = wave_max(m);
    if constexpr (KIND != RDK_PROB_F32) {
        const float to = fminf(fmaxf(wave_m, -a.limit), a.limit) * a.c;
        s = s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f(ref - to);
    }
    const float wave_s = wave_sum(s);
    if (lane_id() == 0) {
        sh.wave_m[wid] = wave_m;
        sh.wave_s[wid] = wave_s;
    }
    sh.keys[tid] = order_key(m) >> 16;
    __syncthreads();
    SoftStat stat{none, 0.f};
    for (int w = 0; w < kWaves; ++w) stat.m = fmaxf(stat.m, sh.wave_m[w]);
    if constexpr (KIND == RDK_PROB_F32) {
        for (int w = 0; w < kWaves; ++w) stat.s += sh.wave_s[w];
    } else {
        const float held = fminf(fmaxf(stat.m, -a.limit), a.limit), to = held * a.c;
        for (int w = 0; w < kWaves; ++w) {
            const float from = fminf(fmaxf(sh.wave_m[w], -a.limit), a.limit) * a.c;
            stat.s += sh.wave_s[w] == 0.f ? 0.f : sh.wave_s[w] * __builtin_amdgcn_exp2f(from - to);
        }
        stat.s *= __builtin_amdgcn_exp2f(-fmaf(held, a.c, -to));   // the rounding of the reference itself
    }
    const bool slow_sum = stat.s != stat.s || (stat.m > -INFINITY && fabsf(stat.m) > a.limit);   // a NaN, or values whose exponents leave the range
    if (wid == 0) {
        uint32_t own[kWaves];
#pragma unroll
        for (int i = 0; i < kWaves; ++i) own[i] = sh.keys[i * kWave + lane_id()];
        const float bound = bound_of<KIND>(own, a.k);
        if (tid == 0) sh.tau = bound;
    }
    __syncthreads();
    tau = sh.tau;
    const int queued = sh.queued;
    for (int q = tid; q < min(queued, kQueue); q += kTopThreads) {
        const int i = begin + (int)sh.queue[q] * V::kLen;
        float v[V::kLen];
        V::to(V::load(xr, i, end), v);
#pragma unroll
        for (int e = 0; e < V::kLen; ++e)
            if (v[e] >= tau) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kQueue) sh.found[at] = entry_of(order_key(v[e]), (uint32_t)(i + e));
            }
    }
    __syncthreads();
    int n = sh.count;
    const uint64_t *sorted = sh.slow.sorted;
    if (slow_sum || queued > kQueue || n > kQueue) {
        n = slow_part<KIND>(a, xr, begin, end, sh, &stat);
    } else {
        n = min(n, a.k);
        sort_found(sh.found, sh.count, a.k, sh.slow.sorted);
        __syncthreads();
    }
    if (a.entries) {
        if (tid < a.k) a.entries[(row * a.parts + part) * a.k + tid] = tid < n ? sorted[tid] : 0;
        if (tid == 0) a.stat[row * a.parts + part] = stat;
        return;
    }
    write_row<KIND>(a.ids, a.values, a.lse, a.k, a.inv_t, row, sorted, n, stat);
}

// Partial statistics of a row brought together, by every lane of a wavefront alike.
template <int KIND>
__device__ __forceinline__ SoftStat merge_stats(const SoftStat *stat, int parts, float c)
{
    SoftStat r{KIND == RDK_PROB_F32 ? 0.f : -INFINITY, 0.f};
    for (int p = 0; p < parts; ++p) r.m = fmaxf(r.m, stat[p].m);
    for (int p = 0; p < parts; ++p) {
        const SoftStat o = stat[p];
        if (KIND == RDK_PROB_F32) r.s += o.s;
        else r.s += o.s == 0.f ? 0.f : o.s * __builtin_amdgcn_exp2f((weight_reference(o.m) - weight_reference(r.m)) * c);
    }
    return r;
}

// The k largest of `count` entries in LDS (0: none), in sh.slow.sorted, by the same bound.  Returns how many there are.
__device__ __forceinline__ int select_entries(const uint64_t *entries, int count, int k, TopShared &sh)
{
    const int tid = threadIdx.x, wid = tid / kWave;
    uint32_t best = 0;
    for (int i = tid; i < count; i += kTopThreads) best = max(best, entry_key(entries[i]));
    sh.keys[tid] = best >> 16;
    if (tid == 0) sh.count = 0;
    __syncthreads();
    if (wid == 0) {
        uint32_t own[kTopThreads / kWave], found = 0;
#pragma unroll
        for (int i = 0; i < kTopThreads / kWave; ++i) own[i] = sh.keys[i * kWave + lane_id()];
#pragma unroll
        for (int bit = 15; bit >= 0; --bit) {
            const uint32_t tried = found | (1u << bit);
            int n = 0;
#pragma unroll
            for (int i = 0; i < kTopThreads / kWave; ++i) n += __popcll(__ballot(own[i] >= tried));
            if (n >= k) found = tried;
        }
        if (tid == 0) sh.queued = (int)found;
    }
    __syncthreads();
    const uint64_t least = max((uint64_t)(uint32_t)sh.queued << 48, (uint64_t)1);
    for (int i = tid; i < count; i += kTopThreads) {
        const uint64_t e = entries[i];
        if (e >= least) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kQueue) sh.found[at] = e;
        }
    }
    __syncthreads();
    const int n = sh.count;
    if (n > kQueue) return select_exact<kTopThreads>([&](int64_t i) { return entries[i]; }, count, k, sh.slow);
    sort_found(sh.found, n, k, sh.slow.sorted);
    __syncthreads();
    return min(n, k);
}

struct TopMergeArgs {
    const uint64_t *entries;
    const SoftStat *stat;
    int k, parts;
    float inv_t, c;
    int32_t *ids;
    float *values, *lse;
};

// The parts of a row brought together.
template <int KIND>
__global__ __launch_bounds__(kTopThreads) void topk_merge_kernel(TopMergeArgs a)
{
    __shared__ TopShared sh;
    __shared__ uint64_t entries[kMergeEntries];
    const int64_t row = blockIdx.x;
    const int count = a.parts * a.k;
    for (int i = threadIdx.x; i < count; i += kTopThreads) entries[i] = a.entries[row * count + i];
    __syncthreads();
    const int n = select_entries(entries, count, a.k, sh);
    write_row<KIND>(a.ids, a.values, a.lse, a.k, a.inv_t, row, sh.slow.sorted, n, merge_stats<KIND>(a.stat + row * a.parts, a.parts, a.c));
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

// One request: scores of its beams' candidates, and the K best of them.
template <int KIND>
__global__ __launch_bounds__(kTopThreads) void beam_merge_kernel(BeamArgs a)
{
    __shared__ TopShared sh;
    __shared__ float beam_m[kWave], beam_log[kWave], beam_score[kWave];
    __shared__ int beam_state[kWave];        // 0: no candidates, 1: finished, 2: live
    extern __shared__ uint64_t scored[];     // [W, parts, k]
    const int64_t g = blockIdx.x, b0 = g * a.W;
    const int tid = threadIdx.x, per = a.parts * a.k, count = a.W * per;
    if (tid < a.W) {
        const float score = a.scores[b0 + tid];
        const int state = score == -INFINITY ? 0 : a.finished && a.finished[b0 + tid] ? 1 : 2;
        beam_score[tid] = score;
        beam_state[tid] = state;
        if (state == 2) {
            const SoftStat st = merge_stats<KIND>(a.stat + (b0 + tid) * a.parts, a.parts, kLog2e);
            beam_m[tid] = weight_reference(st.m);
            beam_log[tid] = KIND == RDK_PROB_F32 ? st.s : logf(st.s);
        }
    }
    __syncthreads();
    for (int i = tid; i < count; i += kTopThreads) {
        const int w = i / per, state = beam_state[w];
        uint64_t e = 0;
        if (state == 1) {
            if (i == w * per) e = entry_of(order_key(beam_score[w]), (uint32_t)w * a.N + a.eos);
        } else if (state == 2 && (e = a.entries[b0 * per + i]) != 0) {
            const float x = key_value(entry_key(e));
            const float score = beam_score[w] + (KIND == RDK_PROB_F32 ? logf(x / beam_log[w]) : (x - beam_m[w]) - beam_log[w]);
            e = score == -INFINITY ? 0 : entry_of(order_key(score), (uint32_t)w * a.N + entry_id(e));
        }
        scored[i] = e;
    }
    __syncthreads();
    const int n = select_entries(scored, count, a.K, sh);
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

// In how many parts a row is read, so that a batch of few rows fills the chip.
int parts_of(int64_t rows, int N, int most)
{
    const int want = (int)((1024 + rows - 1) / rows), maxs = (N + 4095) / 4096;
    int p = want < maxs ? want : maxs;
    p = p < most ? p : most;
    return p < 1 ? 1 : p;
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

TopArgs part_args(RowInput x, int N, int k, int parts, float temperature)
{
    TopArgs a{};
    a.x = x.ptr; a.ldx = x.ld; a.N = N; a.k = k; a.parts = parts;
    a.part_len = (int)align_up(((size_t)N + parts - 1) / parts, 64);
    a.inv_t = 1.f / temperature;
    a.c = a.inv_t * kLog2e;
    a.limit = 1.2676506e30f / (a.c > 1.f ? a.c : 1.f);   // 2^100: the product with c stays in range
    return a;
}

}  // namespace

int select_max_entries() { return kMaxTop; }
int select_max_ids() { return 1 << 30; }   // places in a row, a round of loads behind its end among them, are 32-bit numbers

static int topk_parts(const rdk_topk_desc_t &d) { return parts_of(d.B, d.N, kMergeEntries / d.k); }

size_t topk_workspace_bytes(const rdk_topk_desc_t &d, rdk_input_kind_t kind)
{
    const int parts = topk_parts(d);
    size_t bytes = 0;
    if (parts > 1) carve(d.B, parts, d.k, nullptr, &bytes);
    return bytes;
}

rdk_status_t launch_topk(const rdk_topk_desc_t &d, RowInput x, int32_t *ids, float *values, float *lse, void *ws, hipStream_t st)
{
    const int parts = topk_parts(d);
    TopArgs a = part_args(x, d.N, d.k, parts, d.temperature);
    a.ids = ids; a.values = values; a.lse = lse;
    if (parts > 1) {
        const TopWs w = carve(d.B, parts, d.k, ws, nullptr);
        a.entries = w.entries;
        a.stat = w.stat;
    }
    with_kind(x.kind, [&](auto kind) {
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<decltype(kind)::value>), dim3((unsigned)d.B * parts), dim3(kTopThreads), 0, st, a);
        if (parts > 1) {
            const TopMergeArgs m{a.entries, a.stat, d.k, parts, a.inv_t, a.c, ids, values, lse};
            RDK_TIMED_LAUNCH("topk_merge_kernel", (topk_merge_kernel<decltype(kind)::value>), dim3((unsigned)d.B), dim3(kTopThreads), 0, st, m);
        }
    });
    RDK_LAUNCH_CHECK("topk_part_kernel");
    return RDK_OK;
}

static int beam_parts(const rdk_beam_desc_t &d, int k)
{
    const int most = kBeamEntries / (d.W * k);
    return parts_of((int64_t)d.G * d.W, d.N, most < 1 ? 1 : most);
}

size_t beam_select_workspace_bytes(const rdk_beam_desc_t &d, rdk_input_kind_t kind)
{
    const int k = d.K < d.N ? d.K : d.N;
    size_t bytes = 0;
    carve((int64_t)d.G * d.W, beam_parts(d, k), k, nullptr, &bytes);
    return bytes;
}

rdk_status_t launch_beam_select(const rdk_beam_desc_t &d, RowInput x, const float *scores, const uint8_t *finished, float *scores_out,
                                int32_t *parent, int32_t *token, uint8_t *finished_out, void *ws, hipStream_t st)
{
    const int k = d.K < d.N ? d.K : d.N, parts = beam_parts(d, k);
    const TopWs w = carve((int64_t)d.G * d.W, parts, k, ws, nullptr);
    TopArgs a = part_args(x, d.N, k, parts, 1.f);
    a.scores = scores; a.finished = finished;
    a.entries = w.entries; a.stat = w.stat;
    BeamArgs b{};
    b.entries = w.entries; b.stat = w.stat; b.scores = scores; b.finished = finished;
    b.W = d.W; b.N = d.N; b.k = k; b.K = d.K; b.parts = parts; b.eos = d.eos;
    b.scores_out = scores_out; b.parent = parent; b.token = token; b.finished_out = finished_out;
    rdk_status_t rc = RDK_OK;
    with_kind(x.kind, [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        static LdsGrant grant;
        rc = grant((const void *)&beam_merge_kernel<KIND>, kMaxTop * kWave * sizeof(uint64_t));
        if (rc != RDK_OK) return;
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<KIND>), dim3((unsigned)(d.G * d.W) * parts), dim3(kTopThreads), 0, st, a);
        RDK_TIMED_LAUNCH("beam_merge_kernel", (beam_merge_kernel<KIND>), dim3((unsigned)d.G), dim3(kTopThreads),
                         (size_t)d.W * parts * k * sizeof(uint64_t), st, b);
    });
    if (rc != RDK_OK) return rc;
    RDK_LAUNCH_CHECK("beam_merge_kernel");
    return RDK_OK;
}

}  // namespace rdk
