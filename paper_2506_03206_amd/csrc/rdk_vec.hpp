// Sixteen bytes of a row at a time: eight bf16 or four fp32 values, at any multiple of the element's size.
#pragma once
#include "rdk_device.hpp"

namespace rdk {

// The largest of three as one instruction (fmaxf of values taken apart from bit patterns costs two more, which would quiet signalling NaN: a NaN
// among the operands shows in the sums that every user forms beside it).
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int KIND>
struct Vec {
    static constexpr int kSize = KIND == RDK_LOGIT_BF16 ? 2 : 4;
    static constexpr int kLen = 16 / kSize;   // elements
    // what stands for "no element": -inf for logits, 0 for weights
    static constexpr unsigned kFill = KIND == RDK_LOGIT_BF16 ? 0xFF80u : KIND == RDK_LOGIT_F32 ? 0xFF800000u : 0u;
    static constexpr unsigned kFillWord = KIND == RDK_LOGIT_BF16 ? 0xFF80FF80u : kFill;

    static __device__ __forceinline__ u32x4 fill() { return u32x4{kFillWord, kFillWord, kFillWord, kFillWord}; }

    static __device__ __forceinline__ void to(const u32x4 r, float (&v)[kLen])
    {
        if constexpr (KIND == RDK_LOGIT_BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(r[i] << 16);
                v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
        }
    }

    // What was made of a vector so far is made anew after this: values kept from one pass over a row in registers to the next would take
    // twice the registers of the row itself.
    static __device__ __forceinline__ void again(u32x4 &r)
    {
        if constexpr (KIND == RDK_LOGIT_BF16) asm volatile("" : "+v"(r));
    }

    static __device__ __forceinline__ unsigned one(const void *row, int64_t i)
    {
        if constexpr (KIND == RDK_LOGIT_BF16) return ((const uint16_t *)row)[i];
        return ((const unsigned *)row)[i];
    }

    // The vector `off` bytes behind a place that all lanes share (a scalar base and 32 bits of a lane's own: two registers less per address),
    // of which `left` elements belong to the row: the others are fill.
    static __device__ __forceinline__ u32x4 load_at(const void *base, uint32_t off, int left)
    {
        const char *p = (const char *)base + off;
        if (left >= kLen) return *(const u32x4_any *)p;
        u32x4 r = fill();
#pragma unroll
        for (int e = 0; e < kLen - 1; ++e)   // the vector is not whole
            if (e < left) set(r, e, one(p, e));
        return r;
    }

    // the largest element and m
    static __device__ __forceinline__ float largest(const float (&v)[kLen], float m)
    {
#pragma unroll
        for (int e = 0; e < kLen; e += 2) m = max3(v[e], v[e + 1], m);
        return m;
    }

    // elements i .. i + kLen - 1 of a row that ends at `end`
    static __device__ __forceinline__ u32x4 load(const void *row, int64_t i, int64_t end)
    {
        return load_at((const char *)row + i * kSize, 0, end - i < kLen ? (int)(end - i) : kLen);
    }

    // element e (a constant after unrolling) of a vector
    static __device__ __forceinline__ void set(u32x4 &r, int e, unsigned bits)
    {
        if constexpr (KIND == RDK_LOGIT_BF16)
            r[e / 2] = e % 2 ? (r[e / 2] & 0xFFFFu) | (bits << 16) : (r[e / 2] & 0xFFFF0000u) | bits;
        else
            r[e] = bits;
    }

    // the elements whose bit is set become fill
    static __device__ __forceinline__ void strike(u32x4 &r, unsigned bits)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned m;
            if constexpr (KIND == RDK_LOGIT_BF16)
                m = __builtin_amdgcn_perm((unsigned)__builtin_amdgcn_sbfe((int)bits, 2 * i + 1, 1), (unsigned)__builtin_amdgcn_sbfe((int)bits, 2 * i, 1),
                                          0x05040100u);
            else
                m = (unsigned)__builtin_amdgcn_sbfe((int)bits, i, 1);
            r[i] = (r[i] & ~m) | (kFillWord & m);
        }
    }

    // results in the row's own type, to the nearest, ties to even
    static __device__ __forceinline__ u32x4 from(const float (&v)[kLen])
    {
        u32x4 r;
        if constexpr (KIND == RDK_LOGIT_BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // one conversion instruction for two
                typedef float f2 __attribute__((ext_vector_type(2)));
                typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                r[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(f2{v[2 * i], v[2 * i + 1]}, b2));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
        }
        return r;
    }

    static __device__ __forceinline__ uint16_t round_bf16(float x)
    {
        return __builtin_bit_cast(uint16_t, (__bf16)x);
    }

    // non-temporal: results are larger than the caches, and what is read again should stay there
    static __device__ __forceinline__ void store_at(void *base, uint32_t off, int left, const u32x4 r)
    {
        char *p = (char *)base + off;
        if (left >= kLen) {
            __builtin_nontemporal_store(r, (u32x4_any *)p);
            return;
        }
#pragma unroll
        for (int e = 0; e < kLen - 1; ++e)
            if (e < left) {
                if constexpr (KIND == RDK_LOGIT_BF16) ((uint16_t *)p)[e] = (uint16_t)(r[e / 2] >> (e % 2 * 16));
                else ((unsigned *)p)[e] = r[e];
            }
    }
    static __device__ __forceinline__ void store(void *row, int64_t i, int64_t end, const u32x4 r)
    {
        store_at((char *)row + i * kSize, 0, end - i < kLen ? (int)(end - i) : kLen, r);
    }

    static __device__ __forceinline__ void store1(void *row, int64_t i, float x)
    {
        if constexpr (KIND == RDK_LOGIT_BF16) ((uint16_t *)row)[i] = round_bf16(x);
        else ((float *)row)[i] = x;
    }
};

}  // namespace rdk
