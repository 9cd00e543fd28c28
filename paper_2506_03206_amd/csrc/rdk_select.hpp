// Selection of the largest entries: an order on (value, id) pairs as 64-bit numbers, and the exact k largest of a set by a workgroup.
#pragma once
#include "rdk_device.hpp"

namespace rdk {

constexpr int kMaxTop = 128;   // entries kept per row or request

// A number whose order as an unsigned integer is that of the values: NaN above everything, -0 = +0.
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.f);   // -0 becomes +0
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key)
{
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
constexpr uint32_t kKeyMinusInf = 0x007FFFFFu, kKeyZero = 0x80000000u;

// What stands at or below this is masked: logits of -inf, weights of 0 (and less).
template <int KIND>
__device__ __forceinline__ uint32_t masked_key() { return KIND == RDK_PROB_F32 ? kKeyZero : kKeyMinusInf; }

// The order in which entries are kept: larger values first, of equal ones the lower id.  0 is no entry.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, uint32_t id) { return ((uint64_t)key << 32) | (uint32_t)~id; }
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ uint32_t entry_id(uint64_t e) { return ~(uint32_t)e; }

struct SelectShared {
    uint64_t list[kMaxTop], sorted[kMaxTop];
    int count, wave[16];
};

// The k largest of a workgroup's entries (distinct, 0 for none) into sh.sorted, descending; returns how many there are.  each(f) calls f with every
// entry of the calling thread.  By halving: the k-th largest entry is found bit by bit, with a pass over the set for each, so it is right for
// any set and slow.
template <int THREADS, class Each>
__device__ __forceinline__ int select_exact(const Each &each, int k, SelectShared &sh)
{
    const int wid = threadIdx.x / kWave;
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t tried = least | ((uint64_t)1 << bit);
        int c = 0;
        each([&](uint64_t e) { c += e >= tried; });
        c = (int)wave_sum((float)c);       // counts above 2^24 lose their last bits, where only "at least k" matters
        __syncthreads();                   // sh.wave has been read
        if (lane_id() == 0) sh.wave[wid] = c;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < THREADS / kWave; ++w) total += min(sh.wave[w], k);
        if (total >= k) least = tried;
    }
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    each([&](uint64_t e) {
        if (e != 0 && e >= least) sh.list[atomicAdd(&sh.count, 1)] = e;   // entries are distinct: at most k
    });
    __syncthreads();
    const int n = sh.count;
    if ((int)threadIdx.x < n) {
        const uint64_t own = sh.list[threadIdx.x];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh.list[j] > own;
        sh.sorted[rank] = own;
    }
    __syncthreads();
    return n;
}

}  // namespace rdk
