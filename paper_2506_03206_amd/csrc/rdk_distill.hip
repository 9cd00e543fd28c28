// Distillation of a drafter over its kept slots from its teacher's top logits: the loss of every position and its gradient.
//
// With s = softmax(z / T) and the teacher's probabilities t on the slots A of its entries:  loss = sum_A t (log t - log s), and where the teacher's
// remainder r is counted too, + r (log r - log rho) with rho = sum of s outside A.  Gradient:  (s - t) / T on A,  s (1 - r / rho) / T outside.
// rho is summed over the slots outside A by themselves (a bitmap of A in LDS): as 1 - sum_A s it would be lost to rounding for a drafter
// that is sure of its top entries.
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kMaxEntries = 128;          // teacher entries of a position: two to a lane of one wavefront
constexpr int kPerLane = kMaxEntries / kWave;
constexpr int kDistillThreads = 256;
constexpr int kPartSlots = 65536;         // at most, of a row in one workgroup: the bitmap of A
constexpr float kLog2e = 1.44269504088896341f;

struct DistillArgs {
    const void *z;
    int64_t ldz;
    const int32_t *slot_of;   // target id -> slot, or NULL: ids are slots
    int ids;                  // ids below this have an entry there
    int n, K, parts, part_slots;
    float inv_t;
    const int32_t *top_ids;
    const float *top_logits, *teacher_lse, *weight;
    float *loss;
    float4 *stats;            // reference of the exponents, 1 / sum, coefficient of s outside A, constant of t
    SoftStat *part;           // [B, parts]
    void *dz;
    int64_t ldd;
};

// The teacher's entries of a row, lane l of a wavefront holding the entries l and l + 64; slot -1 for entries that do not count.
struct Entries {
    int slot[kPerLane];
    float v[kPerLane];
};
__device__ __forceinline__ Entries row_entries(const DistillArgs &a, int64_t row)
{
    Entries t;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
        const int k = lane_id() + j * kWave;
        t.slot[j] = -1;
        t.v[j] = -INFINITY;
        if (k < a.K) {
            const int id = a.top_ids[row * a.K + k];
            t.v[j] = a.top_logits[row * a.K + k];
            if (id >= 0 && id < a.ids && t.v[j] != -INFINITY) t.slot[j] = a.slot_of ? max(a.slot_of[id], -1) : id;
        }
    }
    return t;
}

__device__ __forceinline__ float soft_term(float z, float ref, float c) { return __builtin_amdgcn_exp2f((z - ref) * c); }

__device__ __forceinline__ SoftStat merge_at(SoftStat a, SoftStat b, float c)
{
    SoftStat r;
    r.m = fmaxf(a.m, b.m);
    const float ref = weight_reference(r.m);
    r.s = (a.s == 0.f ? 0.f : a.s * soft_term(weight_reference(a.m), ref, c)) + (b.s == 0.f ? 0.f : b.s * soft_term(weight_reference(b.m), ref, c));
    return r;
}

__device__ __forceinline__ SoftStat wave_merge_at(SoftStat v, float c)
{
    SoftStat r;
    r.m = wave_max(v.m);
    r.s = wave_sum(v.s == 0.f ? 0.f : v.s * soft_term(weight_reference(v.m), weight_reference(r.m), c));
    return r;
}

// Statistics of a part of a row; REST: of the slots outside A alone.
template <int KIND, bool REST>
__global__ __launch_bounds__(kDistillThreads) void distill_part_kernel(DistillArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kWaves = kDistillThreads / kWave;
    __shared__ unsigned marked[REST ? kPartSlots / 32 : 1];
    __shared__ SoftStat sh[kWaves];
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * a.part_slots, end = min(a.n, begin + a.part_slots);
    if (a.weight && a.weight[row] == 0.f) return;
    const void *zr = row_ptr<KIND>(a.z, a.ldz, row);
    const float c = a.inv_t * kLog2e;
    if (REST) {
        for (int i = threadIdx.x; i < a.part_slots / 32; i += kDistillThreads) marked[i] = 0;
        __syncthreads();
        if (threadIdx.x < kWave) {
            const Entries t = row_entries(a, row);
#pragma unroll
            for (int j = 0; j < kPerLane; ++j)
                if (t.slot[j] >= begin && t.slot[j] < end) atomicOr(&marked[(t.slot[j] - begin) / 32], 1u << ((t.slot[j] - begin) % 32));
        }
        __syncthreads();
    }
    SoftStat st{-INFINITY, 0.f};
    for (int i = begin + (int)threadIdx.x * V::kLen; i < end; i += kDistillThreads * V::kLen) {
        float v[V::kLen];
        V::to(V::load(zr, i, end), v);
        if (REST) {
            const unsigned bits = marked[(i - begin) / 32] >> ((i - begin) % 32);
#pragma unroll
            for (int e = 0; e < V::kLen; ++e)
                if (bits >> e & 1u) v[e] = -INFINITY;
        }
        float mx = st.m;
#pragma unroll
        for (int e = 0; e < V::kLen; ++e) mx = fmaxf(mx, v[e]);
        const float ref = weight_reference(mx);
        float s = st.s == 0.f ? 0.f : st.s * soft_term(weight_reference(st.m), ref, c);
#pragma unroll
        for (int e = 0; e < V::kLen; ++e) s += soft_term(v[e], ref, c);
        st.m = mx;
        st.s = s;
    }
    st = wave_merge_at(st, c);
    if (lane_id() == 0) sh[threadIdx.x / kWave] = st;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) st = merge_at(st, sh[w], c);
        a.part[row * a.parts + part] = st;
    }
}

// What the row's loss and gradient follow from, by one wavefront: `st` the statistics of the row (REST: of its slots outside A), zt its logits at
// the entries (-inf for those that do not count).  Returns the row's loss without its weight; stats in every lane.
template <bool REST>
__device__ __forceinline__ float row_loss(const DistillArgs &a, int64_t row, const Entries &t, const float (&zt)[kPerLane], SoftStat st, float4 *stats)
{
    const float c = a.inv_t * kLog2e;
    float m = st.m;
    int held = 0;
    float vmax = -INFINITY;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
        if (REST) m = fmaxf(m, zt[j]);
        held += __popcll(__ballot(t.slot[j] >= 0));
        if (t.slot[j] >= 0) vmax = fmaxf(vmax, t.v[j]);
    }
    if (REST) m = wave_max(m);
    vmax = weight_reference(wave_max(vmax));
    const float ref = weight_reference(m);
    float rest = st.s == 0.f ? 0.f : st.s * soft_term(weight_reference(st.m), ref, c), sum_a = 0.f, sum_t = 0.f;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
        if (t.slot[j] >= 0) {
            if (REST) sum_a += soft_term(zt[j], ref, c);
            sum_t += expf((t.v[j] - vmax) * a.inv_t);
        }
    const float total = REST ? rest + wave_sum(sum_a) : rest;
    sum_t = wave_sum(sum_t);
    const bool remainder = REST && held < a.n;
    const float log_total = logf(total);
    // log t = v / T - constant
    const float constant = remainder ? a.teacher_lse[row] : vmax * a.inv_t + logf(sum_t);
    float loss = 0.f, mass = 0.f;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
        if (t.slot[j] >= 0) {
            const float log_t = t.v[j] * a.inv_t - constant, p = expf(log_t);
            const float log_s = total == 0.f ? -INFINITY : (zt[j] - ref) * a.inv_t - log_total;
            mass += p;
            if (p != 0.f) loss += p * (log_t - log_s);
        }
    loss = wave_sum(loss);
    float outside = held ? 1.f : 0.f;
    if (remainder) {
        const float r = fmaxf(0.f, 1.f - wave_sum(mass));
        if (r > 0.f) loss += r * (logf(r) - (rest == 0.f ? -INFINITY : logf(rest) - log_total));
        outside = rest == 0.f ? 1.f : 1.f - r * total / rest;
    }
    *stats = make_float4(ref, total == 0.f ? 0.f : 1.f / total, outside, constant);
    return loss;
}

// The row's logits at the entries.
template <int KIND>
__device__ __forceinline__ void entry_logits(const void *zr, const Entries &t, float (&zt)[kPerLane])
{
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) zt[j] = t.slot[j] >= 0 ? load1<KIND>(zr, t.slot[j]) : -INFINITY;
}

template <int KIND, bool REST>
__global__ __launch_bounds__(kWave) void distill_finish_kernel(DistillArgs a)
{
    const int64_t row = blockIdx.x;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (threadIdx.x == 0) {
            a.loss[row] = 0.f;
            a.stats[row] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return;
    }
    const Entries t = row_entries(a, row);
    float zt[kPerLane];
    entry_logits<KIND>(row_ptr<KIND>(a.z, a.ldz, row), t, zt);
    const float c = a.inv_t * kLog2e;
    SoftStat st{-INFINITY, 0.f};
    for (int p = lane_id(); p < a.parts; p += kWave) st = merge_at(st, a.part[row * a.parts + p], c);
    st = wave_merge_at(st, c);
    float4 stats;
    const float loss = row_loss<REST>(a, row, t, zt, st, &stats);
    if (threadIdx.x == 0) {
        a.loss[row] = w * loss;
        a.stats[row] = stats;
    }
}

// dz of a part of a row.
template <int KIND>
__global__ __launch_bounds__(kDistillThreads) void distill_grad_kernel(DistillArgs a)
{
    typedef Vec<KIND> V;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * a.part_slots, end = min(a.n, begin + a.part_slots);
    const void *zr = row_ptr<KIND>(a.z, a.ldz, row);
    void *dr = const_cast<void *>(row_ptr<KIND>(a.dz, a.ldd, row));
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        const u32x4 zero{0, 0, 0, 0};
        for (int i = begin + (int)threadIdx.x * V::kLen; i < end; i += kDistillThreads * V::kLen) V::store(dr, i, end, zero);
        return;
    }
    const float4 stats = a.stats[row];
    const float c = a.inv_t * kLog2e, wt = w * a.inv_t, scale = stats.y * stats.z * wt;
    Entries t;
    float zt[kPerLane];
    if (threadIdx.x < kWave) {
        t = row_entries(a, row);
        entry_logits<KIND>(zr, t, zt);
    }
    __syncthreads();   // the logits at the entries have been read before anything is written: dz may be z
    for (int i = begin + (int)threadIdx.x * V::kLen; i < end; i += kDistillThreads * V::kLen) {
        float v[V::kLen];
        V::to(V::load(zr, i, end), v);
#pragma unroll
        for (int e = 0; e < V::kLen; ++e) v[e] = scale * soft_term(v[e], stats.x, c);
        V::store(dr, i, end, V::from(v));
    }
    __syncthreads();   // the entries' own gradient goes over what stands at their slots
    if (threadIdx.x < kWave) {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
            if (t.slot[j] >= begin && t.slot[j] < end)
                V::store1(dr, t.slot[j], wt * (soft_term(zt[j], stats.x, c) * stats.y - expf(t.v[j] * a.inv_t - stats.w)));
    }
}

template <class F>
void with_logits(rdk_input_kind_t kind, const F &f)
{
    if (kind == RDK_LOGIT_F32) f(std::integral_constant<int, RDK_LOGIT_F32>());
    else f(std::integral_constant<int, RDK_LOGIT_BF16>());
}

void split(const rdk_distill_desc_t &d, DistillArgs &a)
{
    a.parts = (d.n + kPartSlots - 1) / kPartSlots;
    a.part_slots = (int)align_up((size_t)(d.n + a.parts - 1) / a.parts, 32);
}

DistillArgs arguments(const rdk_distill_desc_t &d, const KernelHandle *h, RowInput z, const int32_t *top_ids, const float *top_logits,
                      const float *weight)
{
    DistillArgs a{};
    a.z = z.ptr; a.ldz = z.ld;
    a.slot_of = h ? h->slot_of : nullptr;
    a.ids = h ? h->N : d.n;
    a.n = d.n; a.K = d.K; a.inv_t = 1.f / d.temperature;
    a.top_ids = top_ids; a.top_logits = top_logits; a.weight = weight;
    split(d, a);
    return a;
}

rdk_status_t launch_grad(const DistillArgs &a, rdk_input_kind_t kind, int32_t B, hipStream_t st)
{
    with_logits(kind, [&](auto k) {
        RDK_TIMED_LAUNCH("distill_grad_kernel", (distill_grad_kernel<decltype(k)::value>), dim3((unsigned)B * a.parts), dim3(kDistillThreads), 0, st, a);
    });
    RDK_LAUNCH_CHECK("distill_grad_kernel");
    return RDK_OK;
}

}  // namespace

int distill_max_entries() { return kMaxEntries; }

size_t distill_workspace_bytes(const rdk_distill_desc_t &d, rdk_input_kind_t kind)
{
    DistillArgs a{};
    split(d, a);
    return align_up((size_t)d.B * a.parts * sizeof(SoftStat), 256) + align_up((size_t)d.B * sizeof(float4), 256);
}

rdk_status_t launch_distill_loss(const rdk_distill_desc_t &d, const KernelHandle *h, RowInput z, const int32_t *top_ids, const float *top_logits,
                                 const float *teacher_lse, const float *weight, float *loss, float *stats, void *dz, int64_t ldd, void *ws,
                                 hipStream_t st)
{
    DistillArgs a = arguments(d, h, z, top_ids, top_logits, weight);
    a.teacher_lse = teacher_lse;
    a.loss = loss;
    a.part = (SoftStat *)ws;
    a.stats = stats ? (float4 *)stats : (float4 *)((char *)ws + align_up((size_t)d.B * a.parts * sizeof(SoftStat), 256));
    a.dz = dz; a.ldd = ldd;
    with_logits(z.kind, [&](auto k) {
        constexpr int KIND = decltype(k)::value;
        if (teacher_lse) {
            RDK_TIMED_LAUNCH("distill_part_kernel", (distill_part_kernel<KIND, true>), dim3((unsigned)d.B * a.parts), dim3(kDistillThreads), 0, st, a);
            RDK_TIMED_LAUNCH("distill_finish_kernel", (distill_finish_kernel<KIND, true>), dim3((unsigned)d.B), dim3(kWave), 0, st, a);
        } else {
            RDK_TIMED_LAUNCH("distill_part_kernel", (distill_part_kernel<KIND, false>), dim3((unsigned)d.B * a.parts), dim3(kDistillThreads), 0, st, a);
            RDK_TIMED_LAUNCH("distill_finish_kernel", (distill_finish_kernel<KIND, false>), dim3((unsigned)d.B), dim3(kWave), 0, st, a);
        }
    });
    RDK_LAUNCH_CHECK("distill_finish_kernel");
    return dz ? launch_grad(a, z.kind, d.B, st) : RDK_OK;
}

rdk_status_t launch_distill_grad(const rdk_distill_desc_t &d, const KernelHandle *h, RowInput z, const int32_t *top_ids, const float *top_logits,
                                 const float *stats, const float *weight, void *dz, int64_t ldd, hipStream_t st)
{
    DistillArgs a = arguments(d, h, z, top_ids, top_logits, weight);
    a.stats = (float4 *)const_cast<float *>(stats);
    a.dz = dz; a.ldd = ldd;
    return launch_grad(a, z.kind, d.B, st);
}

}  // namespace rdk
