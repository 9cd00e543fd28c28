// Distillation of a drafter over its kept slots from its teacher's top logits: the loss of every position and its gradient.
//
// With s = softmax(z / T) and the teacher's probabilities t on the slots A of its entries:  loss = sum_A t (log t - log s), and where the teacher's
// remainder r is counted too, + r (log r - log rho) with rho = sum of s outside A.  Gradient:  (s - t) / T on A,  s (1 - r / rho) / T outside.
// rho is summed over the slots outside A by themselves (a bitmap of A in LDS): as 1 - sum_A s it would be lost to rounding for a drafter
// that is sure of its top entries.  Of a drafter surer still (88 T between its best logit and all outside) it is nothing that fp32 holds beside the row's sum: the
// sum outside is then relative to the largest logit outside, log rho is formed of the two references in 64 bits, and the gradient outside is s - r times the softmax
// over these slots alone.
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kMaxEntries = 128;          // teacher entries of a position: two to a lane of one wavefront
constexpr int kPerLane = kMaxEntries / kWave;
constexpr int kDistillThreads = 256;
constexpr int kGradVecs = 8;             // 16-byte vectors of a thread in the backward call
constexpr int kLoopThreads = 448, kLoopVecs = 4;   // a row read in rounds
constexpr int kPartVecs = 8;             // of a part of a row that several workgroups share
constexpr float kLog2e = 1.44269504088896341f;

struct DistillArgs {
    const void *z;
    int64_t ldz;
    const int32_t *slot_of;   // target id -> slot, or NULL: ids are slots
    int ids;                  // ids below this have an entry there
    int n, K, parts, grad_parts, in_place;
    float inv_t;
    const int32_t *top_ids;
    const float *top_logits, *teacher_lse, *weight;
    float *loss;
    float4 *stats;            // what stats_of() says
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

// The same with the slots known.
__device__ __forceinline__ Entries row_entries(const DistillArgs &a, int64_t row, const int *slots)
{
    Entries t;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
        const int k = lane_id() + j * kWave;
        t.slot[j] = slots[k];
        t.v[j] = k < a.K ? a.top_logits[row * a.K + k] : -INFINITY;
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

// Statistics of a part of a row, whose logits lie in the registers; REST: of the slots outside A alone.  For few rows, whose chain it shortens:
// the loss of 64 bf16 rows of 128256 takes 10.3 us with the launch that joins the parts, where one workgroup a row takes 15.9.
template <int KIND, bool REST>
__global__ __launch_bounds__(kDistillThreads + kWave) void distill_part_kernel(DistillArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kWaves = kDistillThreads / kWave, kSlots = kDistillThreads * kPartVecs * V::kLen;
    __shared__ __attribute__((aligned(16))) uint8_t marked[REST ? kDistillThreads * kPartVecs : 16];
    __shared__ SoftStat sh[kWaves];
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, begin = part * kSlots, here = min(a.n - begin, kSlots), tid = threadIdx.x;
    if (a.weight && a.weight[row] == 0.f) return;
    const char *zr = (const char *)row_ptr<KIND>(a.z, a.ldz, row) + (int64_t)begin * V::kSize;
    const float c = a.inv_t * kLog2e;
    u32x4 raw[kPartVecs];
    if (tid >= kDistillThreads) {
        if (REST) {
            const Entries t = row_entries(a, row);
            for (int i = lane_id() * 16; i < kDistillThreads * kPartVecs; i += kWave * 16) *(u32x4 *)(marked + i) = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < kPerLane; ++j)
                if (t.slot[j] >= begin && t.slot[j] < begin + here) {
                    const int q = (t.slot[j] - begin) / V::kLen, at = q % kDistillThreads * kPartVecs + q / kDistillThreads;
                    atomicOr((unsigned *)marked + at / 4, 1u << (at % 4 * 8 + (t.slot[j] - begin) % V::kLen));
                }
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPartVecs; ++j) {
            const int left = here - (j * kDistillThreads + tid) * V::kLen;
            raw[j] = left > 0 ? V::load_at(zr + j * kDistillThreads * 16, tid * 16, left) : V::fill();
        }
    }
    if (REST) __syncthreads();
    if (tid < kDistillThreads) {
        float v[V::kLen];
        SoftStat st{-INFINITY, 0.f};
#pragma unroll
        for (int j = 0; j < kPartVecs; ++j) {
            if (REST) {
                const unsigned bits = marked[tid * kPartVecs + j];
                if (bits) V::strike(raw[j], bits);
            }
            V::to(raw[j], v);
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) st.m = fmaxf(st.m, v[e]);
        }
        const float ref = weight_reference(st.m);
#pragma unroll
        for (int j = 0; j < kPartVecs; ++j) {
            V::again(raw[j]);
            V::to(raw[j], v);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < V::kLen; ++e) sum += soft_term(v[e], ref, c);
            st.s += sum;
        }
        st = wave_merge_at(st, c);
        if (lane_id() == 0) sh[tid / kWave] = st;
    }
    __syncthreads();
    if (tid == 0) {
        SoftStat st = sh[0];
        for (int w = 1; w < kWaves; ++w) st = merge_at(st, sh[w], c);
        a.part[row * a.parts + part] = st;
    }
}

// The row's logits at the entries.
template <int KIND>
__device__ __forceinline__ void entry_logits(const void *zr, const Entries &t, float (&zt)[kPerLane])
{
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) zt[j] = t.slot[j] >= 0 ? load1<KIND>(zr, t.slot[j]) : -INFINITY;
}

// What the teacher's entries of a row amount to, by one wavefront.  The few sums and logarithms of a row that its loss is a small difference of are
// held in 64 bits.
struct Teacher {
    double log_t[kPerLane];    // log t of the lane's entries
    float p[kPerLane];         // t, 0 for entries that do not count
    double shift;              // log t = (v - the largest v that counts) / T - shift: a number of ordinary size wherever the logits lie
    int held;
    bool remainder;            // the mass outside A counts
    double r;                  // the teacher's
};

// The largest teacher logit that counts.
__device__ __forceinline__ float largest_logit(const Entries &t)
{
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
        if (t.slot[j] >= 0) m = fmaxf(m, t.v[j]);
    return weight_reference(wave_max(m));
}

template <bool REST>
__device__ __forceinline__ Teacher teacher_of(const DistillArgs &a, int64_t row, const Entries &t)
{
    Teacher o;
    o.held = 0;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) o.held += __popcll(__ballot(t.slot[j] >= 0));
    const float vmax = largest_logit(t);
    o.remainder = REST && o.held < a.n;
    if (o.remainder) {
        o.shift = a.teacher_lse[row] - (double)vmax * a.inv_t;
    } else {
        double sum = 0.;
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
            if (t.slot[j] >= 0) sum += expf((t.v[j] - vmax) * a.inv_t);
        o.shift = log(wave_sum(sum));
    }
    double mass = 0.;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
        o.log_t[j] = ((double)t.v[j] - vmax) * a.inv_t - o.shift;
        o.p[j] = t.slot[j] >= 0 ? expf((float)o.log_t[j]) : 0.f;
        mass += o.p[j];
    }
    mass = wave_sum(mass);
    o.r = o.remainder ? fmax(0., 1. - mass) : 0.;
    if (mass != mass) o.r = mass;
    return o;
}

// exp((z - reference) / T) summed over the entries, and their largest logit.
__device__ __forceinline__ SoftStat entry_stat(const Entries &t, const float (&zt)[kPerLane], float c)
{
    SoftStat st;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) m = fmaxf(m, zt[j]);
    st.m = wave_max(m);
    const float ref = weight_reference(st.m);
    st.s = 0.f;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
        if (t.slot[j] >= 0) st.s += soft_term(zt[j], ref, c);
    st.s = wave_sum(st.s);
    return st;
}

// A row's sums brought together.
struct RowSums {
    float ref, total, inv;   // the row's largest logit, its sum relative to that, and the reciprocal
    float out_ref, rest;     // the sum of the slots outside A (without the remainder: of the row) and what it is relative to
    float down;              // exp((out_ref - ref) / T)
    bool far;                // out_ref is not ref
};

// Outside A exponentials are relative to the row's largest logit, of which rho is a quotient with the row's sum (of a drafter near its teacher the errors of
// the two cancel in the loss), unless all outside lies more than kFar powers of two below, which leaves 62 for them in fp32's range.  Then they are
// relative to the largest logit outside.
constexpr float kFar = 64.f;
__device__ __forceinline__ RowSums sums_of(const SoftStat *outside, int parts, SoftStat entries, float c)
{
    RowSums u;
    float top = -INFINITY;
    for (int k = 0; k < parts; ++k) top = fmaxf(top, outside[k].m);
    u.ref = weight_reference(fmaxf(top, entries.m));
    u.far = top > -INFINITY && (top - u.ref) * c < -kFar;
    u.out_ref = u.far ? top : u.ref;
    u.down = u.far ? soft_term(top, u.ref, c) : 1.f;
    u.rest = 0.f;
    for (int k = 0; k < parts; ++k)
        u.rest += outside[k].s == 0.f ? 0.f : outside[k].s * soft_term(weight_reference(outside[k].m), u.out_ref, c);
    u.total = u.rest * u.down + (entries.s == 0.f ? 0.f : entries.s * soft_term(weight_reference(entries.m), u.ref, c));
    u.inv = u.total == 0.f ? 0.f : 1.f / u.total;
    return u;
}

// Factor of exp((z - out_ref) / T) outside A in the gradient.
__device__ __forceinline__ float outside_of(bool remainder, float r, int held, const RowSums &u)
{
    if (!remainder) return held ? u.inv : 0.f;
    if (u.rest == 0.f) return 0.f;
    return u.far ? u.down * u.inv - r / u.rest : u.inv * (1.f - r * u.total / u.rest);
}

// What the backward call reads of a row: a reference of exponents, 1 / the row's sum, the factor of exp((z - reference) / T) outside A, the teacher's shift.
// Where the reference is not the row's largest logit, 1 / sum is relative to the largest logit at the entries and has its sign turned.  A row of weight 0,
// which the forward call does not look at, has a factor that no other row has.
__device__ __forceinline__ float4 passed_over() { return make_float4(0.f, 0.f, -INFINITY, 0.f); }
__device__ __forceinline__ float4 stats_of(const Teacher &o, const RowSums &u)
{
    return make_float4(u.out_ref, u.far ? -u.inv : u.inv, outside_of(o.remainder, (float)o.r, o.held, u), (float)o.shift);
}

// The row's loss, by one wavefront.
__device__ __forceinline__ double loss_of(const DistillArgs &a, const Entries &t, const float (&zt)[kPerLane], const Teacher &o, const RowSums &u)
{
    const double log_total = log((double)u.total);
    double loss = 0.;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
        if (o.p[j] != 0.f) {
            const double log_s = u.total == 0.f ? -INFINITY : ((double)zt[j] - u.ref) * a.inv_t - log_total;
            loss += o.p[j] * (o.log_t[j] - log_s);
        }
    loss = wave_sum(loss);
    if (o.remainder && o.r != 0.) {
        double log_ratio = log(o.r * u.total / u.rest);
        if (u.far) log_ratio -= ((double)u.out_ref - u.ref) * a.inv_t;
        loss += u.rest == 0.f ? INFINITY : o.r * log_ratio;
    }
    return loss;
}

template <int KIND, bool REST>
__global__ __launch_bounds__(kWave) void distill_finish_kernel(DistillArgs a)
{
    const int64_t row = blockIdx.x;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (threadIdx.x == 0) {
            a.loss[row] = 0.f;
            a.stats[row] = passed_over();
        }
        return;
    }
    const Entries t = row_entries(a, row);
    float zt[kPerLane];
    entry_logits<KIND>(row_ptr<KIND>(a.z, a.ldz, row), t, zt);
    const float c = a.inv_t * kLog2e;
    const Teacher o = teacher_of<REST>(a, row, t);
    SoftStat st{-INFINITY, 0.f};
    for (int p = lane_id(); p < a.parts; p += kWave) st = merge_at(st, a.part[row * a.parts + p], c);
    st = wave_merge_at(st, c);
    const RowSums u = sums_of(&st, 1, REST ? entry_stat(t, zt, c) : SoftStat{-INFINITY, 0.f}, c);
    const double loss = loss_of(a, t, zt, o, u);
    if (threadIdx.x == 0) {
        a.loss[row] = (float)(w * loss);
        a.stats[row] = stats_of(o, u);
    }
}

// A row's entries between the steps of the wavefront that follows them.
struct EntryShared {
    double log_t[kMaxEntries], shift, r;
    int slot[kMaxEntries], held, remainder;
    float zt[kMaxEntries], p[kMaxEntries];

    __device__ __forceinline__ void put(const float (&z)[kPerLane], const Teacher &o)
    {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            const int k = lane_id() + j * kWave;
            log_t[k] = o.log_t[j]; zt[k] = z[j]; p[k] = o.p[j];
        }
        if (lane_id() == 0) {
            shift = o.shift; r = o.r; held = o.held; remainder = o.remainder;
        }
    }
    __device__ __forceinline__ void get(Entries &t, float (&z)[kPerLane], Teacher &o) const
    {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            const int k = lane_id() + j * kWave;
            o.log_t[j] = log_t[k]; t.slot[j] = slot[k]; z[j] = zt[k]; o.p[j] = p[k];
        }
        o.shift = shift; o.r = r; o.held = held; o.remainder = remainder;
    }
};

template <int KIND, bool REST>
__device__ __forceinline__ void follow(const DistillArgs &a, int64_t row, const void *zr, float c, const Entries &t, EntryShared &kept, SoftStat *entries)
{
    float zt[kPerLane];
    entry_logits<KIND>(zr, t, zt);
    const Teacher o = teacher_of<REST>(a, row, t);
    if (REST) {
        const SoftStat st = entry_stat(t, zt, c);
        if (lane_id() == 0) *entries = st;
    }
    kept.put(zt, o);
}

// A whole row in the registers of one workgroup: its logits are read once, for the loss and the gradient.  One wavefront beside the THREADS that
// hold the row follows the teacher's entries (ids to slots to logits, a chain of three reads that would otherwise wait for the row: loads
// return in order) and adds up the loss; the entries' own gradient goes over what stands at their slots.
// The exponentials, relative to the largest logit of their thread, stay in the registers for the gradient where 72 of them hold a thread's share
// (the vector unit would be busy with them twice: 19 instructions a logit instead of 12, half as long as the row takes to stream), else
// they are formed again: with seventeen vectors a thread (512 fp32 rows of 61000 54.3 us, 59.6 with them kept), and for bf16 rows in 960 threads
// where no bits of A take registers too (1024 rows of 61000 52.9, kept 56.7; remainder counted 70.1, kept 63.3).  The up to kLen - 1 logits
// behind the last whole vector of a row are one thread's each.
// Bound by HBM where rows are many: loss and gradient of 2048 bf16 rows of 32064 (an eighth of them of weight 0), 64 entries, 45 us = 5.5
// TB/s read and written.  Batches that the chip holds at once load, compute and store one after the other: the loss of 1024 bf16 rows of 16384 takes
// 13 us, of which the loads could be 5 and the vector unit 4.  Few rows are the chain of their entries: 3.9 us for 16 rows of 256.
template <int KIND, int THREADS, int VECS, bool REST, bool GRAD>
__global__ __launch_bounds__(THREADS + kWave) void distill_row_kernel(DistillArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kWaves = THREADS / kWave;
    constexpr bool KEEP = GRAD && VECS * V::kLen <= 72 && (VECS < 17) && (THREADS < 960 || KIND == RDK_LOGIT_F32 || REST);
    constexpr int kMarks = REST ? (int)((THREADS * VECS + 31) / 16 * 16) : 16;
    __shared__ __attribute__((aligned(16))) uint8_t marked[kMarks];   // a bit per slot of A, by the thread that holds it
    __shared__ SoftStat waves[kWaves], entries;
    __shared__ EntryShared kept;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, whole = a.n / V::kLen, behind = a.n % V::kLen;   // whole vectors, logits behind them
    const bool follows = tid >= THREADS;                                          // the wavefront of the entries
    const void *zr = row_ptr<KIND>(a.z, a.ldz, row);
    void *dr = GRAD ? const_cast<void *>(row_ptr<KIND>(a.dz, a.ldd, row)) : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (GRAD) {
            const u32x4 zero{0, 0, 0, 0};
            for (int i = tid * V::kLen; i < a.n; i += (THREADS + kWave) * V::kLen) V::store(dr, i, a.n, zero);
        }
        if (tid == 0) {
            a.loss[row] = 0.f;
            if (a.stats) a.stats[row] = passed_over();
        }
        return;
    }
    const float c = a.inv_t * kLog2e;
    u32x4 raw[VECS];
    float last = -INFINITY;
    if (follows) {
        const Entries t = row_entries(a, row);
        if (REST) {
            for (int i = lane_id() * 16; i < kMarks; i += kWave * 16) *(u32x4 *)(marked + i) = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < kPerLane; ++j)
                if (t.slot[j] >= 0) {
                    const int q = t.slot[j] / V::kLen, at = q == whole ? THREADS * VECS : q % THREADS * VECS + q / THREADS;
                    atomicOr((unsigned *)marked + at / 4, 1u << (at % 4 * 8 + t.slot[j] % V::kLen));
                }
        }
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) kept.slot[lane_id() + j * kWave] = t.slot[j];
        if (!REST) follow<KIND, REST>(a, row, zr, c, t, kept, &entries);
    } else {
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            raw[j] = V::fill();
            if (j * THREADS + tid < whole) raw[j] = *(const u32x4_any *)((const char *)zr + j * THREADS * 16 + (uint32_t)tid * 16);
        }
        if (tid < behind) last = load1<KIND>(zr, whole * V::kLen + tid);
    }
    if (REST) {
        __syncthreads();
        if (follows) {
            const Entries t = row_entries(a, row, kept.slot);
            follow<KIND, REST>(a, row, zr, c, t, kept, &entries);
        } else {
#pragma unroll
            for (int j = 0; j < VECS; ++j) {
                const unsigned bits = marked[tid * VECS + j];
                if (bits) V::strike(raw[j], bits);
            }
            if (tid < behind && (marked[THREADS * VECS] >> tid & 1)) last = -INFINITY;
        }
    }
    float v[V::kLen], e[KEEP ? VECS : 1][V::kLen], own_ref = 0.f, own_s = 0.f, e_last = 0.f;
    if (!follows) {
        float m = last;
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            V::to(raw[j], v);
#pragma unroll
            for (int k = 0; k < V::kLen; ++k) m = fmaxf(m, v[k]);
        }
        own_ref = weight_reference(m);
        own_s = e_last = soft_term(last, own_ref, c);
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            V::again(raw[j]);
            V::to(raw[j], v);
            float part = 0.f;
#pragma unroll
            for (int k = 0; k < V::kLen; ++k) {
                const float x = soft_term(v[k], own_ref, c);
                if (KEEP) e[j][k] = x;
                part += x;
            }
            own_s += part;
        }
        const SoftStat st = wave_merge_at(SoftStat{m, own_s}, c);
        if (lane_id() == 0) waves[tid / kWave] = st;
    }
    __syncthreads();   // (the logits at the entries have been read too: dz may be z)
    const RowSums u = sums_of(waves, kWaves, REST ? entries : SoftStat{-INFINITY, 0.f}, c);
    const float wt = w * a.inv_t;
    if (GRAD) {
        const float scale = wt * outside_of(REST && kept.remainder, (float)kept.r, kept.held, u);
        const float own_scale = own_s == 0.f ? 0.f : scale * soft_term(own_ref, u.out_ref, c);
        if (!follows) {
#pragma unroll
            for (int j = 0; j < VECS; ++j)
                if (j * THREADS + tid < whole) {
                    if (!KEEP) {
                        V::again(raw[j]);
                        V::to(raw[j], v);
                    }
#pragma unroll
                    for (int k = 0; k < V::kLen; ++k) v[k] = KEEP ? own_scale * e[j][k] : scale * soft_term(v[k], u.out_ref, c);
                    V::store_at((char *)dr + j * THREADS * 16, tid * 16, V::kLen, V::from(v));
                }
            if (tid < behind) V::store1(dr, whole * V::kLen + tid, own_scale * e_last);
        }
    }
    Entries t;
    float zt[kPerLane];
    Teacher o;
    if (follows) {
        kept.get(t, zt, o);
        const double loss = loss_of(a, t, zt, o, u);
        if (lane_id() == 0) {
            a.loss[row] = (float)(w * loss);
            if (a.stats) a.stats[row] = stats_of(o, u);
        }
    }
    if (!GRAD) return;
    __syncthreads();
    if (follows) {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
            if (t.slot[j] >= 0) V::store1(dr, t.slot[j], wt * (soft_term(zt[j], u.ref, c) * u.inv - o.p[j]));
    }
}

// The loss of a row too long for the registers, or for enough workgroups with it there, read in rounds by one workgroup; the bits of A for the whole
// row in dynamic LDS.  512 bf16 rows of 128256, remainder counted: 29 us = 4.5 TB/s; 1024 of 50000 22.4 us = 4.6 TB/s.
template <int KIND, bool REST>
__global__ __launch_bounds__(kLoopThreads + kWave) void distill_loop_kernel(DistillArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kWaves = kLoopThreads / kWave, kRound = kLoopThreads * kLoopVecs;   // vectors
    extern __shared__ __attribute__((aligned(16))) uint8_t marked_row[];               // a byte per vector of the row
    __shared__ SoftStat waves[kWaves], entries;
    __shared__ EntryShared kept;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, vectors = (a.n + V::kLen - 1) / V::kLen;
    const bool follows = tid >= kLoopThreads;
    const char *zr = (const char *)row_ptr<KIND>(a.z, a.ldz, row);
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (tid == 0) {
            a.loss[row] = 0.f;
            a.stats[row] = passed_over();
        }
        return;
    }
    const float c = a.inv_t * kLog2e;
    const int whole = a.n / V::kLen, behind = a.n % V::kLen;   // whole vectors (there are some: rows are long), logits behind them
    // Always as many loads, of the last vector where the round has none of its own: the compiler counts loads in flight, and would wait for all of
    // them behind a branch that has some of its own.
    auto load_round = [&](u32x4 (&raw)[kLoopVecs], int base) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoopVecs; ++j)
            raw[j] = *(const u32x4_any *)(zr + (uint64_t)(uint32_t)min(base + j * kLoopThreads + tid, whole - 1) * 16);
    };
    u32x4 raw[kLoopVecs], ahead[kLoopVecs];
    float last = -INFINITY;
    if (!follows) {
        load_round(raw, 0);
        if (tid < behind) last = load1<KIND>(zr, whole * V::kLen + tid);
    }
    if (REST) {
        for (int i = tid * 16; i < vectors; i += (kLoopThreads + kWave) * 16) *(u32x4 *)(marked_row + i) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    if (follows) {
        const Entries t = row_entries(a, row);
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            if (REST && t.slot[j] >= 0) {
                const int at = t.slot[j] / V::kLen;
                atomicOr((unsigned *)marked_row + at / 4, 1u << (at % 4 * 8 + t.slot[j] % V::kLen));
            }
            kept.slot[lane_id() + j * kWave] = t.slot[j];
        }
    }
    if (REST) __syncthreads();
    if (follows) {
        const Entries t = row_entries(a, row, kept.slot);
        follow<KIND, REST>(a, row, zr, c, t, kept, &entries);
    } else {
        if (REST && tid < behind && (marked_row[whole] >> tid & 1)) last = -INFINITY;
        SoftStat st{last, last == -INFINITY ? 0.f : 1.f};
        if (last != last) st.s = last;
        auto take_round = [&](u32x4 (&now)[kLoopVecs], int base) __attribute__((always_inline)) {
            float v[V::kLen], m = st.m;
#pragma unroll
            for (int j = 0; j < kLoopVecs; ++j) {
                const int at = base + j * kLoopThreads + tid;
                if (at >= whole) now[j] = V::fill();
                if (REST && at < whole) {
                    const unsigned bits = marked_row[at];
                    if (bits) V::strike(now[j], bits);
                }
                V::to(now[j], v);
                m = V::largest(v, m);
            }
            const float ref = weight_reference(m);
            float sum = st.s == 0.f ? 0.f : st.s * soft_term(weight_reference(st.m), ref, c);
#pragma unroll
            for (int j = 0; j < kLoopVecs; ++j) {
                V::again(now[j]);
                V::to(now[j], v);
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < V::kLen; ++e) part += soft_term(v[e], ref, c);
                sum += part;
            }
            st = SoftStat{m, sum};
        };
#pragma unroll 1
        for (int base = 0;; base += 2 * kRound) {
            load_round(ahead, base + kRound);
            take_round(raw, base);
            if (base + kRound >= whole) break;
            load_round(raw, base + 2 * kRound);
            take_round(ahead, base + kRound);
            if (base + 2 * kRound >= whole) break;
        }
        st = wave_merge_at(st, c);
        if (lane_id() == 0) waves[tid / kWave] = st;
    }
    __syncthreads();
    if (!follows) return;
    SoftStat st = lane_id() < kWaves ? waves[lane_id()] : SoftStat{-INFINITY, 0.f};
    st = wave_merge_at(st, c);
    const RowSums u = sums_of(&st, 1, REST ? entries : SoftStat{-INFINITY, 0.f}, c);
    Entries t;
    float zt[kPerLane];
    Teacher o;
    kept.get(t, zt, o);
    const double loss = loss_of(a, t, zt, o, u);
    if (lane_id() == 0) {
        a.loss[row] = (float)(w * loss);
        a.stats[row] = stats_of(o, u);
    }
}

// dz of a part of a row, whose logits lie in the registers; the entries as in distill_row_kernel.  Bound by HBM: 1024 bf16 rows of
// 16384 (an eighth of weight 0) 8 to 9 us = 7 to 7.8 TB/s read and written.  The L2s fetch z anew (33 MB counted at their far side); the rate, above
// the 6.0 to 6.4 of a copy, says that the last-level cache behind them still has it from the forward call.
// A row of two references (stats_of) needs the logits of all its entries: over z itself they stand only until another workgroup writes its part, so
// the first one goes over the whole of such a row (64 rows of 128256 over z: 33 us if all are of this kind, 7 if none is).
template <int KIND>
__global__ __launch_bounds__(kDistillThreads + kWave) void distill_grad_kernel(DistillArgs a)
{
    typedef Vec<KIND> V;
    constexpr int kSlots = kDistillThreads * kGradVecs * V::kLen;
    const int64_t row = blockIdx.x / a.grad_parts;
    const int part = blockIdx.x % a.grad_parts, begin = part * kSlots, here = min(a.n - begin, kSlots), tid = threadIdx.x;   // (n may be 2^31 - 1)
    const bool follows = tid >= kDistillThreads;
    const char *zr = (const char *)row_ptr<KIND>(a.z, a.ldz, row);
    char *dr = (char *)const_cast<void *>(row_ptr<KIND>(a.dz, a.ldd, row));
    const float w = a.weight ? a.weight[row] : 1.f;
    const float4 stats = a.stats[row];
    if (w == 0.f || stats.z == passed_over().z) {
        const u32x4 zero{0, 0, 0, 0};
        for (int i = tid * V::kLen; i < here; i += (kDistillThreads + kWave) * V::kLen) V::store(dr + (int64_t)begin * V::kSize, i, here, zero);
        return;
    }
    u32x4 raw[kGradVecs];
    Entries t;
    float zt[kPerLane];
    auto load_part = [&](int from) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kGradVecs; ++j) {
            const int left = min(a.n - from, kSlots) - (j * kDistillThreads + tid) * V::kLen;
            raw[j] = left > 0 ? V::load_at(zr + (int64_t)from * V::kSize + j * kDistillThreads * 16, tid * 16, left) : V::fill();
        }
    };
    if (follows) {
        t = row_entries(a, row);
        entry_logits<KIND>(zr, t, zt);
    } else {
        load_part(begin);
    }
    const bool two = stats.y < 0.f, alone = two && a.in_place && a.grad_parts > 1;
    if (alone && part > 0) return;
    const int end = alone ? a.n : begin + here;
    const float c = a.inv_t * kLog2e, wt = w * a.inv_t, scale = stats.z * wt;
    if (a.in_place) __syncthreads();   // the logits at the entries have been read before anything is written
    if (!follows) {
#pragma unroll 1
        for (int from = begin;;) {
#pragma unroll
            for (int j = 0; j < kGradVecs; ++j) {
                const int left = min(a.n - from, kSlots) - (j * kDistillThreads + tid) * V::kLen;
                if (left > 0) {
                    float v[V::kLen];
                    V::to(raw[j], v);
#pragma unroll
                    for (int e = 0; e < V::kLen; ++e) v[e] = scale * soft_term(v[e], stats.x, c);
                    V::store_at(dr + (int64_t)from * V::kSize + j * kDistillThreads * 16, tid * 16, left, V::from(v));
                }
            }
            if (end - from <= kSlots) break;
            from += kSlots;
            load_part(from);
        }
    }
    __syncthreads();
    if (follows) {
        const float vmax = largest_logit(t), ref = two ? weight_reference(wave_max(fmaxf(zt[0], zt[1]))) : stats.x, inv = fabsf(stats.y);
        static_assert(kPerLane == 2, "the largest logit at the entries is formed of two to a lane");
#pragma unroll
        for (int j = 0; j < kPerLane; ++j)
            if (t.slot[j] >= begin && t.slot[j] < end)
                V::store1(dr, t.slot[j], wt * (soft_term(zt[j], ref, c) * inv - expf((t.v[j] - vmax) * a.inv_t - stats.w)));
    }
}

// The longest row that a workgroup holds.
template <int KIND>
constexpr int kRowSlots = 960 * 17 * Vec<KIND>::kLen;

// The longest row read in rounds: its bits of A take 60 KB of LDS.
template <int KIND>
constexpr int kLoopSlots = 60 * 1024 * Vec<KIND>::kLen;

template <class F>
void with_logits(rdk_input_kind_t kind, const F &f)
{
    if (kind == RDK_LOGIT_F32) f(std::integral_constant<int, RDK_LOGIT_F32>());
    else f(std::integral_constant<int, RDK_LOGIT_BF16>());
}

// Parts that several workgroups share a row by.
int parts_of(int n, rdk_input_kind_t kind)
{
    const int slots = kDistillThreads * kPartVecs * (kind == RDK_LOGIT_BF16 ? 8 : 4);
    return (n - 1) / slots + 1;
}

int grad_parts_of(int n, rdk_input_kind_t kind)
{
    const int slots = kDistillThreads * kGradVecs * (kind == RDK_LOGIT_BF16 ? 8 : 4);
    return (n - 1) / slots + 1;
}

DistillArgs arguments(const rdk_distill_desc_t &d, const KernelHandle *h, RowInput z, const int32_t *top_ids, const float *top_logits,
                      const float *weight, void *dz, int64_t ldd)
{
    DistillArgs a{};
    a.z = z.ptr; a.ldz = z.ld;
    a.slot_of = h ? h->slot_of : nullptr;
    a.ids = h ? h->N : d.n;
    a.n = d.n; a.K = d.K; a.inv_t = 1.f / d.temperature;
    a.top_ids = top_ids; a.top_logits = top_logits; a.weight = weight;
    a.parts = parts_of(d.n, z.kind);
    a.grad_parts = grad_parts_of(d.n, z.kind);
    a.dz = dz; a.ldd = ldd;
    a.in_place = dz == z.ptr;
    return a;
}

template <int KIND>
rdk_status_t launch_grad(const DistillArgs &a, int32_t B, hipStream_t st)
{
    RDK_TIMED_LAUNCH("distill_grad_kernel", (distill_grad_kernel<KIND>), dim3((unsigned)B * a.grad_parts), dim3(kDistillThreads + kWave), 0, st, a);
    RDK_LAUNCH_CHECK("distill_grad_kernel");
    return RDK_OK;
}

template <int KIND, bool REST>
rdk_status_t launch_split(const DistillArgs &a, int32_t B, hipStream_t st)
{
    RDK_TIMED_LAUNCH("distill_part_kernel", (distill_part_kernel<KIND, REST>), dim3((unsigned)B * a.parts), dim3(kDistillThreads + kWave), 0, st, a);
    RDK_TIMED_LAUNCH("distill_finish_kernel", (distill_finish_kernel<KIND, REST>), dim3((unsigned)B), dim3(kWave), 0, st, a);
    RDK_LAUNCH_CHECK("distill_finish_kernel");
    return a.dz ? launch_grad<KIND>(a, B, st) : RDK_OK;
}

template <int KIND, int THREADS, int VECS, bool REST>
rdk_status_t launch_both(const DistillArgs &a, int32_t B, hipStream_t st)
{
    RDK_TIMED_LAUNCH("distill_row_kernel", (distill_row_kernel<KIND, THREADS, VECS, REST, true>), dim3((unsigned)B), dim3(THREADS + kWave), 0, st, a);
    RDK_LAUNCH_CHECK("distill_row_kernel");
    return RDK_OK;
}

template <int KIND, int THREADS, int VECS, bool REST>
rdk_status_t launch_row(const DistillArgs &a, int32_t B, hipStream_t st)
{
    if (a.dz) return launch_both<KIND, THREADS, VECS, REST>(a, B, st);
    RDK_TIMED_LAUNCH("distill_row_kernel", (distill_row_kernel<KIND, THREADS, VECS, REST, false>), dim3((unsigned)B), dim3(THREADS + kWave), 0, st, a);
    RDK_LAUNCH_CHECK("distill_row_kernel");
    return RDK_OK;
}

template <int KIND, bool REST>
rdk_status_t launch_loop(const DistillArgs &a, int32_t B, hipStream_t st)
{
    const size_t lds = REST ? align_up((size_t)(a.n - 1) / Vec<KIND>::kLen + 1, 16) : 0;
    RDK_TIMED_LAUNCH("distill_loop_kernel", (distill_loop_kernel<KIND, REST>), dim3((unsigned)B), dim3(kLoopThreads + kWave), lds, st, a);
    RDK_LAUNCH_CHECK("distill_loop_kernel");
    return a.dz ? launch_grad<KIND>(a, B, st) : RDK_OK;
}

template <int KIND, bool REST>
rdk_status_t launch_loss(const DistillArgs &a, int32_t B, hipStream_t st)
{
    constexpr int kLen = Vec<KIND>::kLen;
    // Few rows, and long: several workgroups to a row, in one launch more (bf16, remainder counted: the loss of 64 rows of 62000 10.7 -> 8.7 us, of
    // 128256 15.9 -> 10.3; 192 rows 16.8 -> 16.3 and 11.1 -> 12.2; with the gradient 64 rows of 128256 20.7 -> 15.8, 128 rows 22.7 -> 24.4).
    const bool few = a.dz ? B <= (a.n > kRowSlots<KIND> ? 128 : 64) && a.n > 960 * 9 * kLen : B <= 128 && a.n > 448 * 17 * kLen;
    if (few || a.n > kLoopSlots<KIND>) return launch_split<KIND, REST>(a, B, st);
    // The loss alone of rows beyond 64 KB: in rounds, three workgroups on a compute unit where the registers of long rows leave one or two (2048 fp32
    // rows of 32064 88 -> 48 us, 512 bf16 rows of 128256 41 -> 29, 1024 of 50000 28.1 -> 26.7; 2048 bf16 rows of 32064 30.6 -> 33.8 and so not).
    // With the gradient only rows that no workgroup holds, which are then read again.
    if (a.n > (a.dz ? kRowSlots<KIND> : 448 * 9 * kLen)) return launch_loop<KIND, REST>(a, B, st);
    // As many threads and vectors to a thread as the row takes: two workgroups of eight wavefronts on a compute unit for the rows in between (2048 bf16
    // rows of 32064: 448 threads of nine vectors 47.5 us, 512 of eight 62, one workgroup of 960 60), one for the longest.  Beyond nine vectors the
    // exponentials are formed twice: 2048 rows of 32064 and of 32768, all of them counted, 52 and 60 us.
    if (a.n <= 192 * 3 * kLen) return launch_row<KIND, 192, 3, REST>(a, B, st);
    if (a.n <= 192 * 9 * kLen) return launch_row<KIND, 192, 9, REST>(a, B, st);
    if (a.n <= 448 * 5 * kLen) return launch_row<KIND, 448, 5, REST>(a, B, st);
    if (a.n <= 448 * 9 * kLen) return launch_row<KIND, 448, 9, REST>(a, B, st);
    if (a.n <= 448 * 17 * kLen) return launch_both<KIND, 448, 17, REST>(a, B, st);
    if (a.n <= 960 * 9 * kLen) return launch_both<KIND, 960, 9, REST>(a, B, st);
    return launch_both<KIND, 960, 17, REST>(a, B, st);
}

}  // namespace

int distill_max_entries() { return kMaxEntries; }

size_t distill_workspace_bytes(const rdk_distill_desc_t &d, rdk_input_kind_t kind)
{
    return align_up((size_t)d.B * parts_of(d.n, kind) * sizeof(SoftStat), 256) + align_up((size_t)d.B * sizeof(float4), 256);
}

rdk_status_t launch_distill_loss(const rdk_distill_desc_t &d, const KernelHandle *h, RowInput z, const int32_t *top_ids, const float *top_logits,
                                 const float *teacher_lse, const float *weight, float *loss, float *stats, void *dz, int64_t ldd, void *ws,
                                 hipStream_t st)
{
    DistillArgs a = arguments(d, h, z, top_ids, top_logits, weight, dz, ldd);
    a.teacher_lse = teacher_lse;
    a.loss = loss;
    a.part = (SoftStat *)ws;
    a.stats = stats ? (float4 *)stats : (float4 *)((char *)ws + align_up((size_t)d.B * a.parts * sizeof(SoftStat), 256));
    rdk_status_t rc = RDK_OK;
    with_logits(z.kind, [&](auto k) {
        constexpr int KIND = decltype(k)::value;
        rc = teacher_lse ? launch_loss<KIND, true>(a, d.B, st) : launch_loss<KIND, false>(a, d.B, st);
    });
    return rc;
}

rdk_status_t launch_distill_grad(const rdk_distill_desc_t &d, const KernelHandle *h, RowInput z, const int32_t *top_ids, const float *top_logits,
                                 const float *stats, const float *weight, void *dz, int64_t ldd, hipStream_t st)
{
    DistillArgs a = arguments(d, h, z, top_ids, top_logits, weight, dz, ldd);
    a.stats = (float4 *)const_cast<float *>(stats);
    rdk_status_t rc = RDK_OK;
    with_logits(z.kind, [&](auto k) { rc = launch_grad<decltype(k)::value>(a, d.B, st); });
    return rc;
}

}  // namespace rdk
