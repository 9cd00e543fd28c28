// The states of beams after a selection: rows of device buffers copied by an index of parents, in place or from one buffer into another.
//
// A thread owns one unit (up to 16 bytes) of a row's bytes for every beam of a request: it reads the units of all rows that change before it
// writes any of them, so a reorder in place needs no scratch and no order between threads.
#include "rdk_vec.hpp"

namespace rdk {

namespace {

constexpr int kStatesPerLaunch = 24, kReorderThreads = 256, kMaxBeams = 64;

struct StateArg {
    const char *src;
    char *dst;
    int64_t src_stride, dst_stride, src_pitch, dst_pitch;
    int64_t units;          // per row: segments * units per segment
    int64_t per_segment;    // units of a segment
    unsigned first_block;   // of the launch
    unsigned blocks;        // per request
    unsigned unit;          // bytes
};
struct StateArgs {
    StateArg s[kStatesPerLaunch];
    int count, G, W, K, in_place;   // in_place: a bit per state
    const int32_t *parent;
};

template <class T>
__device__ void reorder_unit(const StateArgs &a, const StateArg &s, int64_t g, int64_t u, const int *from)
{
    const int64_t seg = u / s.per_segment, off = (u - seg * s.per_segment) * (int64_t)sizeof(T);
    const char *src = s.src + g * a.W * s.src_stride + seg * s.src_pitch + off;
    char *dst = s.dst + g * a.K * s.dst_stride + seg * s.dst_pitch + off;
    T v[kMaxBeams];
#pragma unroll
    for (int i = 0; i < kMaxBeams; ++i)
        if (i < a.K && from[i] >= 0) v[i] = *(const T *)(src + from[i] * s.src_stride);
#pragma unroll
    for (int i = 0; i < kMaxBeams; ++i)
        if (i < a.K && from[i] >= 0) *(T *)(dst + i * s.dst_stride) = v[i];
}

__global__ __launch_bounds__(kReorderThreads) void beam_reorder_kernel(StateArgs a)
{
    __shared__ int from[kMaxBeams];
    int n = 0;
    while (n + 1 < a.count && blockIdx.x >= a.s[n + 1].first_block) ++n;
    const StateArg &s = a.s[n];
    const unsigned b = blockIdx.x - s.first_block;
    const int64_t g = b / s.blocks, u = (int64_t)(b % s.blocks) * kReorderThreads + threadIdx.x;
    if ((int)threadIdx.x < a.K) {
        const int p = a.parent[g * a.K + threadIdx.x];
        const bool stays = (a.in_place >> n & 1) && p == (int)threadIdx.x;
        from[threadIdx.x] = p < 0 || p >= a.W || stays ? -1 : p;
    }
    __syncthreads();
    if (u >= s.units) return;
    switch (s.unit) {
        case 16: reorder_unit<u32x4>(a, s, g, u, from); break;
        case 8: reorder_unit<uint64_t>(a, s, g, u, from); break;
        case 4: reorder_unit<uint32_t>(a, s, g, u, from); break;
        case 2: reorder_unit<uint16_t>(a, s, g, u, from); break;
        default: reorder_unit<uint8_t>(a, s, g, u, from); break;
    }
}

}  // namespace

int reorder_max_beams() { return kMaxBeams; }

rdk_status_t launch_beam_reorder(int32_t G, int32_t W, int32_t K, const int32_t *parent, const rdk_state_t *states, int32_t count, hipStream_t st)
{
    for (int done = 0; done < count;) {
        StateArgs a{};
        a.G = G; a.W = W; a.K = K; a.parent = parent;
        uint64_t blocks = 0;
        while (done < count && a.count < kStatesPerLaunch) {
            const rdk_state_t &t = states[done];
            if (t.segments == 0 || t.segment_bytes == 0) {   // nothing of it is filled
                ++done;
                continue;
            }
            StateArg s{};
            s.src = (const char *)t.src; s.dst = (char *)t.dst;
            s.src_stride = t.src_stride; s.dst_stride = t.dst_stride;
            s.src_pitch = t.segments > 1 ? t.src_pitch : 0; s.dst_pitch = t.segments > 1 ? t.dst_pitch : 0;
            uint64_t bits = (uintptr_t)t.src | (uintptr_t)t.dst | (uint64_t)t.src_stride | (uint64_t)t.dst_stride | (uint64_t)s.src_pitch |
                            (uint64_t)s.dst_pitch | (uint64_t)t.segment_bytes;
            s.unit = 16;
            while (bits & (s.unit - 1)) s.unit /= 2;
            s.per_segment = t.segment_bytes / s.unit;
            s.units = t.segments * s.per_segment;
            const uint64_t per = ((uint64_t)s.units + kReorderThreads - 1) / kReorderThreads;
            if (a.count && blocks + per * G > 0x7FFFFFFFull) break;
            s.first_block = (unsigned)blocks;
            s.blocks = (unsigned)per;
            blocks += per * G;
            if (t.src == t.dst) a.in_place |= 1 << a.count;
            a.s[a.count++] = s;
            ++done;
        }
        if (!a.count) break;
        RDK_TIMED_LAUNCH("beam_reorder_kernel", beam_reorder_kernel, dim3((unsigned)blocks), dim3(kReorderThreads), 0, st, a);
        RDK_LAUNCH_CHECK("beam_reorder_kernel");
    }
    return RDK_OK;
}

}  // namespace rdk
