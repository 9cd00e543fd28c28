// The k largest entries of rows over a vocabulary with the logarithm of their normaliser, and beam search's selection over beams and
// vocabulary, which takes the K largest entries of every live beam and merges them per request.
#include "rdk_select.hpp"
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kTopThreads = 256;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

struct TopArgs {
    const void *x;
    int64_t ldx;
    int N, k;
    float inv_t;
    // rows of beams that have no candidates among the ids are passed over
    const float *scores;
    const uint8_t *finished;
    uint64_t *entries;      // [rows, k]
    int *counts;            // [rows]
    SoftStat *stat;         // [rows]
    int32_t *ids;           // or, for topk itself, the outputs
    float *values, *lse;
};

template <int KIND>
__global__ __launch_bounds__(kTopThreads) void topk_part_kernel(TopArgs a)
{
    typedef Vec<KIND> V;
    __shared__ SelectShared sh;
    __shared__ SoftStat part[kTopThreads / kWave];
    const int64_t row = blockIdx.x;
    if (a.finished && a.finished[row]) return;
    if (a.scores && a.scores[row] == -INFINITY) return;
    const void *xr = row_ptr<KIND>(a.x, a.ldx, row);
    const float c = a.inv_t * kLog2e;
    SoftStat st{KIND == RDK_PROB_F32 ? 0.f : -INFINITY, 0.f};
    for (int64_t i = (int64_t)threadIdx.x * V::kLen; i < a.N; i += (int64_t)kTopThreads * V::kLen) {
        float v[V::kLen];
        V::to(V::load(xr, i, a.N), v);
        if (KIND == RDK_PROB_F32) {
            for (int e = 0; e < V::kLen; ++e) st.s += v[e], st.m = fmaxf(st.m, v[e]);
        } else {
            float mx = st.m;
            for (int e = 0; e < V::kLen; ++e) mx = fmaxf(mx, v[e]);
            const float ref = weight_reference(mx);
            float s = st.s * __builtin_amdgcn_exp2f((weight_reference(st.m) - ref) * c);
            if (st.s == 0.f) s = 0.f;
            for (int e = 0; e < V::kLen; ++e) s += __builtin_amdgcn_exp2f((v[e] - ref) * c);
            st.m = mx;
            st.s = s;
        }
    }
    {
        const float m = wave_max(st.m), ref = weight_reference(m);
        if (KIND != RDK_PROB_F32) st.s = st.s == 0.f ? 0.f : st.s * __builtin_amdgcn_exp2f((weight_reference(st.m) - ref) * c);
        st.s = wave_sum(st.s);
        st.m = m;
        if (lane_id() == 0) part[threadIdx.x / kWave] = st;
        __syncthreads();
        st = part[0];
        for (int w = 1; w < kTopThreads / kWave; ++w) {
            const SoftStat o = part[w];
            if (KIND == RDK_PROB_F32) {
                st.s += o.s;
                st.m = fmaxf(st.m, o.m);
            } else {
                const float mm = fmaxf(st.m, o.m), ref2 = weight_reference(mm);
                st.s = (st.s == 0.f ? 0.f : st.s * __builtin_amdgcn_exp2f((weight_reference(st.m) - ref2) * c)) +
                       (o.s == 0.f ? 0.f : o.s * __builtin_amdgcn_exp2f((weight_reference(o.m) - ref2) * c));
                st.m = mm;
            }
        }
    }
    const uint32_t masked = masked_key<KIND>();
    const int n = select_exact<kTopThreads>(
        [&](int64_t i) {
            const uint32_t key = order_key(load1<KIND>(xr, i));
            return key > masked ? entry_of(key, (uint32_t)i) : 0;
        },
        a.N, a.k, sh);
    if (a.entries) {
        if ((int)threadIdx.x < n) a.entries[row * a.k + threadIdx.x] = sh.sorted[threadIdx.x];
        if (threadIdx.x == 0) {
            a.counts[row] = n;
            a.stat[row] = st;
        }
        return;
    }
    if ((int)threadIdx.x < a.k) {
        const bool in = (int)threadIdx.x < n;
        const uint64_t e = in ? sh.sorted[threadIdx.x] : 0;
        a.ids[row * a.k + threadIdx.x] = in ? (int32_t)entry_id(e) : -1;
        a.values[row * a.k + threadIdx.x] = in ? key_value(entry_key(e)) : KIND == RDK_PROB_F32 ? 0.f : -INFINITY;
    }
    if (a.lse && threadIdx.x == 0)
        a.lse[row] = KIND == RDK_PROB_F32 ? logf(st.s) : st.s == 0.f ? -INFINITY : weight_reference(st.m) * a.inv_t + logf(st.s);
}

struct BeamArgs {
    const uint64_t *entries;
    const int *counts;
    const SoftStat *stat;
    const float *scores;
    const uint8_t *finished;
    int W, N, k, K, eos;
    float *scores_out;
    int32_t *parent, *token;
    uint8_t *finished_out;
};

// One request: scores of its beams' candidates, and the K best of them.
template <int KIND>
__global__ __launch_bounds__(kTopThreads) void beam_merge_kernel(BeamArgs a)
{
    __shared__ SelectShared sh;
    const int64_t g = blockIdx.x, b0 = g * a.W;
    const int n = select_exact<kTopThreads>(
        [&](int64_t i) -> uint64_t {
            const int w = (int)i / a.k, t = (int)i % a.k;
            const float s = a.scores[b0 + w];
            if (a.finished && a.finished[b0 + w])
                return t == 0 && s != -INFINITY ? entry_of(order_key(s), (uint32_t)w * a.N + a.eos) : 0;
            if (s == -INFINITY || t >= a.counts[b0 + w]) return 0;
            const SoftStat st = a.stat[b0 + w];
            const uint64_t e = a.entries[(b0 + w) * a.k + t];
            const float x = key_value(entry_key(e));
            const float lp = KIND == RDK_PROB_F32 ? logf(x / st.s) : (x - weight_reference(st.m)) - logf(st.s);
            const float score = s + lp;
            return score == -INFINITY ? 0 : entry_of(order_key(score), (uint32_t)w * a.N + entry_id(e));
        },
        (int64_t)a.W * a.k, a.K, sh);
    if ((int)threadIdx.x < a.K) {
        const bool in = (int)threadIdx.x < n;
        const uint64_t e = in ? sh.sorted[threadIdx.x] : 0;
        const int w = in ? (int)(entry_id(e) / (uint32_t)a.N) : -1, j = in ? (int)(entry_id(e) % (uint32_t)a.N) : -1;
        const int64_t o = g * a.K + threadIdx.x;
        a.scores_out[o] = in ? key_value(entry_key(e)) : -INFINITY;
        a.parent[o] = w;
        a.token[o] = j;
        if (a.finished_out) a.finished_out[o] = in && (j == a.eos || (a.finished && a.finished[b0 + w]));
    }
}

template <class F>
void with_kind(rdk_input_kind_t kind, const F &f)
{
    if (kind == RDK_PROB_F32) f(std::integral_constant<int, RDK_PROB_F32>());
    else if (kind == RDK_LOGIT_F32) f(std::integral_constant<int, RDK_LOGIT_F32>());
    else f(std::integral_constant<int, RDK_LOGIT_BF16>());
}

struct TopWs {
    uint64_t *entries;
    SoftStat *stat;
    int *counts;
};

TopWs carve(int64_t rows, int k, void *ws, size_t *bytes)
{
    TopWs w;
    char *p = (char *)ws;
    w.entries = (uint64_t *)p; p += align_up((size_t)rows * k * sizeof(uint64_t), 256);
    w.stat = (SoftStat *)p; p += align_up((size_t)rows * sizeof(SoftStat), 256);
    w.counts = (int *)p; p += align_up((size_t)rows * sizeof(int), 256);
    if (bytes) *bytes = (size_t)(p - (char *)ws);
    return w;
}

}  // namespace

int select_max_entries() { return kMaxTop; }

size_t topk_workspace_bytes(const rdk_topk_desc_t &d, rdk_input_kind_t kind) { return 0; }

rdk_status_t launch_topk(const rdk_topk_desc_t &d, RowInput x, int32_t *ids, float *values, float *lse, void *ws, hipStream_t st)
{
    TopArgs a{};
    a.x = x.ptr; a.ldx = x.ld; a.N = d.N; a.k = d.k; a.inv_t = 1.f / d.temperature;
    a.ids = ids; a.values = values; a.lse = lse;
    with_kind(x.kind, [&](auto kind) {
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<decltype(kind)::value>), dim3((unsigned)d.B), dim3(kTopThreads), 0, st, a);
    });
    RDK_LAUNCH_CHECK("topk_part_kernel");
    return RDK_OK;
}

size_t beam_select_workspace_bytes(const rdk_beam_desc_t &d, rdk_input_kind_t kind)
{
    size_t bytes = 0;
    carve((int64_t)d.G * d.W, d.K < d.N ? d.K : d.N, nullptr, &bytes);
    return bytes;
}

rdk_status_t launch_beam_select(const rdk_beam_desc_t &d, RowInput x, const float *scores, const uint8_t *finished, float *scores_out,
                                int32_t *parent, int32_t *token, uint8_t *finished_out, void *ws, hipStream_t st)
{
    const int k = d.K < d.N ? d.K : d.N;
    const TopWs w = carve((int64_t)d.G * d.W, k, ws, nullptr);
    TopArgs a{};
    a.x = x.ptr; a.ldx = x.ld; a.N = d.N; a.k = k; a.inv_t = 1.f;
    a.scores = scores; a.finished = finished;
    a.entries = w.entries; a.counts = w.counts; a.stat = w.stat;
    BeamArgs b{};
    b.entries = w.entries; b.counts = w.counts; b.stat = w.stat; b.scores = scores; b.finished = finished;
    b.W = d.W; b.N = d.N; b.k = k; b.K = d.K; b.eos = d.eos;
    b.scores_out = scores_out; b.parent = parent; b.token = token; b.finished_out = finished_out;
    with_kind(x.kind, [&](auto kind) {
        RDK_TIMED_LAUNCH("topk_part_kernel", (topk_part_kernel<decltype(kind)::value>), dim3((unsigned)(d.G * d.W)), dim3(kTopThreads), 0, st, a);
        RDK_TIMED_LAUNCH("beam_merge_kernel", (beam_merge_kernel<decltype(kind)::value>), dim3((unsigned)d.G), dim3(kTopThreads), 0, st, b);
    });
    RDK_LAUNCH_CHECK("beam_merge_kernel");
    return RDK_OK;
}

}  // namespace rdk
