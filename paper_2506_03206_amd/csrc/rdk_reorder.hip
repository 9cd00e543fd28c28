// The states of beams after a selection: rows of device buffers copied by an index of parents, in place or from one buffer into another.
//
// A thread owns one unit (16 bytes, less at the end of a piece) of a row's bytes for every beam of a request: it reads the units of all rows that
// change before it writes any of them, so a reorder in place needs no scratch and no order between threads.  Units lie at any address
// (the memory pipe takes them: five beams with rows of 8 pieces of 65934 bytes move at 4.3 TB/s, in units as small as the sizes' common
// divisor at 1.4).  Bound by HBM: 5.8 to 6.2 TB/s of the bytes of rows that change and are needed, where a copy kernel reaches 6.0 to 6.4;
// non-temporal accesses are worth an eighth (16 requests of 4 beams, 0.54 GB of caches: 137 us without, 131 stores alone, 119 to 122 both).
#include "rdk_vec.hpp"

namespace rdk {

namespace {

// Units at any address (as members: a template argument would lose the alignment).
struct Unit16 { typedef unsigned type __attribute__((ext_vector_type(4), aligned(1))); };
struct Unit8 { typedef unsigned type __attribute__((ext_vector_type(2), aligned(1))); };
struct Unit4 { typedef unsigned type __attribute__((aligned(1))); };
struct Unit2 { typedef unsigned short type __attribute__((aligned(1))); };
struct Unit1 { typedef unsigned char type; };

// The parents of a request, which nothing writes meanwhile: read by the scalar unit, once for a wavefront.
typedef const __attribute__((address_space(4))) int *Parents;

constexpr int kStatesPerLaunch = 24, kReorderThreads = 256, kMaxBeams = 64;
constexpr unsigned kMostBlocks = 0xFFFFFFFFu / kReorderThreads;   // of a launch: its threads are counted in 32 bits
constexpr unsigned kMostPerRequest = 1u << 20;                    // of a request; longer rows are moved by several launches

struct StateArg {
    const char *src;
    char *dst;
    int64_t src_stride, dst_stride, src_pitch, dst_pitch;
    int64_t units;          // per row: segments * units per segment
    int64_t per_segment;    // units of a segment, the last of which may have less than 16 bytes
    int64_t segment_bytes;
    unsigned first_block;   // of the launch
    unsigned blocks;        // per request
    int first_request;      // of the launch
    int64_t first_unit;
};
struct StateArgs {
    StateArg s[kStatesPerLaunch];
    int count, W, K, in_place;   // in_place: a bit per state
    const int32_t *parent;
};

// The units of the rows I .. MOST - 1: all are read on the way down, and written on the way back up.  (One variable a row: an array of them is
// made one wide register tuple, copied at every branch.)
template <class U, int I, int MOST>
struct Rows {
    typedef typename U::type T;
    static __device__ __forceinline__ void move(const char *src, char *dst, int64_t src_stride, int64_t dst_stride, Parents parent, int W, int K, bool in_place)
    {
        const int p = I < K ? parent[I] : -1;
        const bool moves = (unsigned)p < (unsigned)W && !(in_place && p == I);   // the same for the workgroup
        T v{};   // (unset, four rows take 2 to 3 % longer, in turn on one card: 0.54 GB of caches 128.9 us, set 125.2; eight rows the same)
        if (moves) v = __builtin_nontemporal_load((const T *)(src + p * src_stride));
        Rows<U, I + 1, MOST>::move(src, dst, src_stride, dst_stride, parent, W, K, in_place);
        if (moves) __builtin_nontemporal_store(v, (T *)(dst + I * dst_stride));
    }
};
template <class U, int MOST>
struct Rows<U, MOST, MOST> {
    static __device__ __forceinline__ void move(const char *, char *, int64_t, int64_t, Parents, int, int, bool) {}
};

// MOST: rows held in registers, K or more.
template <int MOST>
__global__ __launch_bounds__(kReorderThreads, MOST <= 8 ? 8 : MOST <= 16 ? 5 : MOST <= 32 ? 3 : 1) void beam_reorder_kernel(StateArgs a)
{
    int n = 0;
    while (n + 1 < a.count && blockIdx.x >= a.s[n + 1].first_block) ++n;
    const StateArg &s = a.s[n];
    const unsigned b = blockIdx.x - s.first_block, request = b / s.blocks;
    const int64_t g = s.first_request + (int64_t)request;
    const Parents parent = (Parents)(a.parent + g * a.K);
    const bool in_place = a.in_place >> n & 1;
    const int64_t u = s.first_unit + (int64_t)(b - request * s.blocks) * kReorderThreads + threadIdx.x;
    if (u >= s.units) return;
    int64_t seg = 0;
    if (s.units != s.per_segment) seg = (s.units >> 32) == 0 ? (uint32_t)u / (uint32_t)s.per_segment : u / s.per_segment;
    const int64_t off = (u - seg * s.per_segment) * 16;
    const char *src = s.src + g * a.W * s.src_stride + seg * s.src_pitch + off;
    char *dst = s.dst + g * a.K * s.dst_stride + seg * s.dst_pitch + off;
    auto move = [&](auto unit, int at) __attribute__((always_inline)) {
        Rows<decltype(unit), 0, MOST>::move(src + at, dst + at, s.src_stride, s.dst_stride, parent, a.W, a.K, in_place);
    };
    const int left = s.segment_bytes - off < 16 ? (int)(s.segment_bytes - off) : 16;
    if (left == 16) {
        move(Unit16(), 0);
        return;
    }
    if (left & 8) move(Unit8(), 0);
    if (left & 4) move(Unit4(), left & 8);
    if (left & 2) move(Unit2(), left & 12);
    if (left & 1) move(Unit1(), left & 14);
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
    int32_t request = 0;   // of the state at hand, the first that no launch has, and its first unit
    int64_t unit = 0;
    for (int done = 0; done < count;) {
        StateArgs a{};
        a.W = W; a.K = K; a.parent = parent;
        unsigned blocks = 0;
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
            s.segment_bytes = t.segment_bytes;
            s.per_segment = (t.segment_bytes + 15) / 16;
            s.units = t.segments * s.per_segment;
            const uint64_t per = ((uint64_t)(s.units - unit) + kReorderThreads - 1) / kReorderThreads;
            s.first_block = blocks;
            s.blocks = per < kMostPerRequest ? (unsigned)per : kMostPerRequest;
            s.first_request = request;
            s.first_unit = unit;
            const unsigned room = (kMostBlocks - blocks) / s.blocks, left = (unsigned)(G - request);
            if (room == 0) break;
            const unsigned requests = left < room ? left : room;
            blocks += requests * s.blocks;
            if (t.src == t.dst) a.in_place |= 1 << a.count;
            a.s[a.count++] = s;
            request += (int32_t)requests;
            if (request == G) {
                request = 0;
                unit += (int64_t)s.blocks * kReorderThreads;
            }
            if (unit >= s.units) {
                unit = 0;
                ++done;
            }
        }
        if (!a.count) break;
        with_rows(K, [&](auto rows) {
            RDK_TIMED_LAUNCH("beam_reorder_kernel", (beam_reorder_kernel<decltype(rows)::value>), dim3(blocks), dim3(kReorderThreads), 0, st, a);
        });
        RDK_LAUNCH_CHECK("beam_reorder_kernel");
    }
    return RDK_OK;
}

}  // namespace rdk
