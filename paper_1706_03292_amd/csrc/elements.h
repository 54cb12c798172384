// Element types of the network-end operators (fp32 and bf16 in memory, fp32 in
// registers), eight neighbours at a time, and the counter-based generator
// behind dropout.
#pragma once

#include "common.h"

namespace poseidon {
namespace {

typedef __bf16 bf8e __attribute__((ext_vector_type(8)));
typedef __bf16 bf8a __attribute__((ext_vector_type(8), aligned(2)));   // 16 bytes at any element boundary
typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
typedef float f4e __attribute__((ext_vector_type(4)));
typedef float f8e __attribute__((ext_vector_type(8)));

constexpr int GROUP = 8;   // neighbours that a thread loads together and that share one generator call

__device__ __forceinline__ void load_group(const float* p, float (&v)[GROUP])
{
    const f4a a = *reinterpret_cast<const f4a*>(p), b = *reinterpret_cast<const f4a*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}

__device__ __forceinline__ void load_group(const __bf16* p, float (&v)[GROUP])
{
    const bf8a a = *reinterpret_cast<const bf8a*>(p);
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        v[i] = static_cast<float>(a[i]);
}

__device__ __forceinline__ void store_group(float* p, const float (&v)[GROUP])
{
    f4a a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = v[i];
        b[i] = v[4 + i];
    }
    *reinterpret_cast<f4a*>(p) = a;
    *reinterpret_cast<f4a*>(p + 4) = b;
}

// Rounded to nearest, once, as the value leaves the registers.
__device__ __forceinline__ void store_group(__bf16* p, const float (&v)[GROUP])
{
    f8e a;
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        a[i] = v[i];
    *reinterpret_cast<bf8a*>(p) = __builtin_convertvector(a, bf8e);
}

// The first n of the group at p; the others read 0 and are not touched.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int64_t n, float (&v)[GROUP])
{
    if (n >= GROUP) {
        load_group(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            v[i] = i < n ? static_cast<float>(p[i]) : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store_some(T* p, int64_t n, const float (&v)[GROUP])
{
    if (n >= GROUP) {
        store_group(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            if (i < n)
                p[i] = static_cast<T>(v[i]);
    }
}

// A group as it lies in memory, for loads that stay in flight while another
// group is worked on.
template <typename T>
struct Raw;
template <>
struct Raw<__bf16> {
    bf8e v;
};
template <>
struct Raw<float> {
    f4e a, b;
};

__device__ __forceinline__ void load_raw(const __bf16* p, int64_t n, Raw<__bf16>& r)
{
    if (n >= GROUP) {
        r.v = *reinterpret_cast<const bf8a*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            r.v[i] = i < n ? p[i] : static_cast<__bf16>(0.f);
    }
}

__device__ __forceinline__ void load_raw(const float* p, int64_t n, Raw<float>& r)
{
    if (n >= GROUP) {
        r.a = *reinterpret_cast<const f4a*>(p);
        r.b = *reinterpret_cast<const f4a*>(p + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.a[i] = i < n ? p[i] : 0.f;
            r.b[i] = 4 + i < n ? p[4 + i] : 0.f;
        }
    }
}

__device__ __forceinline__ float raw_value(const Raw<__bf16>& r, int i) { return static_cast<float>(r.v[i]); }
__device__ __forceinline__ float raw_value(const Raw<float>& r, int i) { return i < 4 ? r.a[i] : r.b[i - 4]; }

// Philox4x32 (Salmon, Moraes, Dror and Shaw, "Parallel Random Numbers: As Easy
// as 1, 2, 3", SC 2011) with seven rounds, the fewest that pass the whole of
// BigCrush there; ten rounds would make the bf16 dropout kernel bound by its
// integer products instead of memory.  Key: the seed.  Counter: the group's
// number and the caller's offset.
struct Rng {
    uint64_t seed, offset;
};

__device__ __forceinline__ void philox(const Rng& r, uint64_t group, uint32_t (&c)[4])
{
    uint32_t k0 = static_cast<uint32_t>(r.seed), k1 = static_cast<uint32_t>(r.seed >> 32);
    c[0] = static_cast<uint32_t>(group);
    c[1] = static_cast<uint32_t>(group >> 32);
    c[2] = static_cast<uint32_t>(r.offset);
    c[3] = static_cast<uint32_t>(r.offset >> 32);
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c[0];
        const uint64_t b = static_cast<uint64_t>(0xCD9E8D57u) * c[2];
        c[0] = static_cast<uint32_t>(b >> 32) ^ c[1] ^ k0;
        c[1] = static_cast<uint32_t>(b);
        c[2] = static_cast<uint32_t>(a >> 32) ^ c[3] ^ k1;
        c[3] = static_cast<uint32_t>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// Dropout of one group: element i is dropped where its 16 bits (the low half
// of word i / 2, then the high half) are below thr, else scaled.  A dropped
// element is replaced, not multiplied by 0, so an infinity or NaN there
// leaves nothing.
__device__ __forceinline__ void drop_group(float (&v)[GROUP], const Rng& r, uint64_t group, uint32_t thr, float scale)
{
    uint32_t w[4];
    philox(r, group, w);
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const uint32_t bits = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
        v[i] = bits < thr ? 0.f : v[i] * scale;
    }
}

}  // namespace
}  // namespace poseidon
