// Shared by the operators around the layer (linear*.hip, dropout.hip, balance.hip).
#pragma once

#include "common.h"

namespace sw {

// Dropout of a tensor's elements: stream 3 of the library's generator, two elements a draw.
struct Drop {
    uint32_t seed_lo, term, thr;   // an element is dropped iff its 16 bits are < thr
    float scale;                   // 2^16 / (2^16 - thr)
    int on;
};
static inline bool drop_rate_ok(float rate) { return rate >= 0.f && rate < 1.f; }
static inline Drop drop_of(float rate, uint64_t seed) {
    Drop d;
    d.seed_lo = (uint32_t)seed;
    d.term = (uint32_t)(seed >> 32) + 3u * 0x7F4A7C15u;
    d.thr = (uint32_t)((double)rate * 65536.0);
    d.scale = (float)(65536.0 / (65536.0 - (double)d.thr));
    d.on = d.thr > 0;
    return d;
}
// The 32 bits of elements 2 pair and 2 pair + 1: low and high half.
__device__ __forceinline__ uint32_t drop_bits(const Drop &d, uint64_t pair) {
    return noise_bits((uint32_t)pair, d.seed_lo, d.term + (uint32_t)(pair >> 32) * 0x632BE5ABu);
}
// v[0 .. N - 1], elements first .. first + N - 1 (first and N even): those dropped become zero
template <int N> __device__ __forceinline__ void drop_apply(const Drop &d, uint64_t first, float *v) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const uint32_t z = drop_bits(d, (first >> 1) + (uint32_t)(i >> 1));
        v[i] = (z & 0xFFFFu) >= d.thr ? v[i] : 0.f;
        v[i + 1] = (z >> 16) >= d.thr ? v[i + 1] : 0.f;
    }
}

// Eight consecutive elements as floats, 16 or 32 bytes of aligned memory.
template <typename T> struct Eight;
template <> struct Eight<bf16> {
    typedef bf16 V __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void load(const bf16 *p, float *v) {
        const V x = *(const V *)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    }
    static __device__ __forceinline__ void store(bf16 *p, const float *v) {
        V x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (bf16)v[i];
        *(V *)p = x;
    }
};
template <> struct Eight<float> {
    typedef float V __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ void load(const float *p, float *v) {
        const V a = *(const V *)p, b = *(const V *)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    }
    static __device__ __forceinline__ void store(float *p, const float *v) {
        *(V *)p = V{v[0], v[1], v[2], v[3]};
        *(V *)(p + 4) = V{v[4], v[5], v[6], v[7]};
    }
};

// 16 bytes of consecutive elements as floats.
template <typename T> struct Row16 {
    static constexpr int n = 16 / sizeof(T);
    static __device__ __forceinline__ void load(const void *p, int64_t at, float *v) {
        if constexpr (n == 8) Eight<T>::load((const T *)p + at, v);
        else *(float4 *)v = *(const float4 *)((const T *)p + at);
    }
    static __device__ __forceinline__ void store(void *p, int64_t at, const float *v) {
        if constexpr (n == 8) Eight<T>::store((T *)p + at, v);
        else *(float4 *)((T *)p + at) = *(const float4 *)v;
    }
};

}  // namespace sw
