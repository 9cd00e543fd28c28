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

// The units of the rows I .. MOST - 1: all are read on the way down, and written on the way back up.  (One variable a row: an array of them is
// made one wide register tuple, copied at every branch.)
template <class T, int I, int MOST>
struct Rows {
    static __device__ __forceinline__ void move(const char *src, char *dst, int64_t src_stride, int64_t dst_stride, const int *parent, int W, int K,
                                                bool in_place)
    {
        const int p = I < K ? parent[I] : -1;
        const bool moves = (unsigned)p < (unsigned)W && !(in_place && p == I);   // the same for the workgroup
        T v{};
        if (moves) v = __builtin_nontemporal_load((const T *)(src + p * src_stride));
        Rows<T, I + 1, MOST>::move(src, dst, src_stride, dst_stride, parent, W, K, in_place);
        if (moves) __builtin_nontemporal_store(v, (T *)(dst + I * dst_stride));
    }
};
template <class T, int MOST>
struct Rows<T, MOST, MOST> {
    static __device__ __forceinline__ void move(const char *, char *, int64_t, int64_t, const int *, int, int, bool) {}
};

// MOST: rows held in registers, K or more.
template <class T, int MOST>
__device__ __forceinline__ void reorder_unit(const StateArgs &a, const StateArg &s, int64_t g, int64_t u, const int *parent, bool in_place)
{
    int64_t seg = 0;
    if (s.units != s.per_segment) seg = (s.units >> 32) == 0 ? (uint32_t)u / (uint32_t)s.per_segment : u / s.per_segment;
    const int64_t off = (u - seg * s.per_segment) * (int64_t)sizeof(T);
    const char *src = s.src + g * a.W * s.src_stride + seg * s.src_pitch + off;
    char *dst = s.dst + g * a.K * s.dst_stride + seg * s.dst_pitch + off;
    Rows<T, 0, MOST>::move(src, dst, s.src_stride, s.dst_stride, parent, a.W, a.K, in_place);
}

template <int MOST>
__global__ __launch_bounds__(kReorderThreads, MOST <= 8 ? 8 : MOST <= 16 ? 5 : MOST <= 32 ? 3 : 1) void beam_reorder_kernel(StateArgs a)
{
    int n = 0;
    while (n + 1 < a.count && blockIdx.x >= a.s[n + 1].first_block) ++n;
    const StateArg &s = a.s[n];
    const unsigned b = blockIdx.x - s.first_block, g = b / s.blocks;
    const int64_t u = (int64_t)(b - g * s.blocks) * kReorderThreads + threadIdx.x;
    if (u >= s.units) return;
    const int *parent = a.parent + (int64_t)g * a.K;
    const bool in_place = a.in_place >> n & 1;
    switch (s.unit) {
        case 16: reorder_unit<u32x4, MOST>(a, s, g, u, parent, in_place); break;
        case 8: reorder_unit<uint64_t, MOST>(a, s, g, u, parent, in_place); break;
        case 4: reorder_unit<uint32_t, MOST>(a, s, g, u, parent, in_place); break;
        case 2: reorder_unit<uint16_t, MOST>(a, s, g, u, parent, in_place); break;
        default: reorder_unit<uint8_t, MOST>(a, s, g, u, parent, in_place); break;
    }
}

template <class F>
void with_rows(int K, const F &f)
{
    if (K <= 4) f(std::integral_constant<int, 4>());
    else if (K <= 8) f(std::integral_constant<int, 8>());
    else if (K <= 16) f(std::integral_constant<int, 16>());
    else if (K <= 32) f(std::integral_constant<int, 32>());
    else f(std::integral_constant<int, 64>());
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
        with_rows(K, [&](auto rows) {
            RDK_TIMED_LAUNCH("beam_reorder_kernel", (beam_reorder_kernel<decltype(rows)::value>), dim3((unsigned)blocks), dim3(kReorderThreads), 0, st, a);
        });
        RDK_LAUNCH_CHECK("beam_reorder_kernel");
    }
    return RDK_OK;
}

}  // namespace rdk
