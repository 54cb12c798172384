// AdamW over many tensors, the gradients' norm, and the values of 8-bit moments
// (include/poseidon.h gives the formulas and the code's layout).  All of it is a
// few operations per value, bound by memory: every array is read once and written
// once.
//
// The tensors' descriptors travel by value in the kernel arguments; a workgroup
// finds its tensor by counting the first blocks that it has reached, and works on
// `chunk` values of it, eight neighbours a thread and turn.
#include <math.h>

#include "elements.h"
#include "optimizer.h"

namespace poseidon {
namespace {

constexpr int THREADS = 256;
static_assert(ADAMW_CHUNK == THREADS * GROUP, "one group a thread");

// The tensor of workgroup b: the number of later tensors whose first block it
// has reached (independent scalar loads instead of a search's chain of them).
__device__ __forceinline__ int tensor_of(const AdamwGroup& a, int b)
{
    int t = 0;
#pragma unroll
    for (int k = 1; k < ADAMW_GROUP; ++k)
        t += (k < a.count && a.first_block[k] <= b) ? 1 : 0;
    return t;
}

// Sum over the workers of the (up to eight) values at g, in 64 bits and in the
// workers' order, four of them in flight.
template <typename T>
__device__ __forceinline__ void sum_workers(const T* g, int64_t stride, int P, int64_t left, double (&s)[GROUP])
{
    Raw<T> r[4];
    load_raw(g, left, r[0]);
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        s[i] = raw_value(r[0], i);
    int p = 1;
    for (; p + 4 <= P; p += 4) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            load_raw(g + (p + c) * stride, left, r[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                s[i] += raw_value(r[c], i);
    }
    for (; p < P; ++p) {
        load_raw(g + p * stride, left, r[0]);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            s[i] += raw_value(r[0], i);
    }
}

// b^t for t >= 1, by squaring: within 2^-46 of it for any t.
__device__ __forceinline__ double power(double b, int64_t t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1) {
        if (t & 1)
            r *= b;
        b *= b;
    }
    return r;
}

// What a step multiplies with, from its rule.
struct Rates {
    double beta1, beta2, one_beta1, one_beta2, lr;
    float eps, rate, root;   // rate = lr / (1 - beta1^t), root = (1 - beta2^t)^-1/2
    const double* clock;
    const float* scale;
    const int64_t* rng;
};

__device__ __forceinline__ void read_clock(Rates& r)
{
    if (!r.clock)
        return;
    r.lr = r.clock[0];
    const double at = r.clock[1];
    const int64_t t = at >= 1.0 ? (at < 9e18 ? static_cast<int64_t>(at) : INT64_MAX) : 1;
    r.rate = static_cast<float>(r.lr / (1.0 - power(r.beta1, t)));
    r.root = static_cast<float>(1.0 / sqrt(1.0 - power(r.beta2, t)));
}

// W - lr (decay W + (m / c1) / (sqrt(v / c2) + eps))
__device__ __forceinline__ float stepped(float w, float m, float v, float decay, const Rates& r)
{
    const float u = r.rate * m / fmaf(sqrtf(v), r.root, r.eps);
    return w - fmaf(decay, w, u);
}

// ---------------------------------------------------------------------------
// The step with fp32 moments.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(THREADS) void step_kernel(const AdamwGroup a, Rates r)
{
    const double scale = r.scale ? *r.scale : 1.f;
    if (!isfinite(scale))
        return;
    read_clock(r);
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const int64_t e = static_cast<int64_t>(blockIdx.x - a.first_block[t]) * ADAMW_CHUNK + threadIdx.x * GROUP;
    const int64_t left = q.n - e;
    if (left <= 0)
        return;
    float* pm = static_cast<float*>(q.m) + e;
    float* pv = static_cast<float*>(q.v) + e;
    double s[GROUP];
    float w[GROUP], m[GROUP], v[GROUP];
    load_some(q.W + e, left, w);
    load_some(pm, left, m);
    load_some(pv, left, v);
    sum_workers(static_cast<const T*>(q.G) + e, q.stride, q.P, left, s);
    const float b1 = static_cast<float>(r.beta1), b2 = static_cast<float>(r.beta2);
    const float o1 = static_cast<float>(r.one_beta1), o2 = static_cast<float>(r.one_beta2);
    const float decay = static_cast<float>(r.lr * q.weight_decay);
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const float g = static_cast<float>(s[i] * scale);
        m[i] = fmaf(b1, m[i], o1 * g);
        v[i] = fmaf(b2, v[i], o2 * (g * g));
        w[i] = stepped(w[i], m[i], v[i], decay, r);
    }
    store_some(q.W + e, left, w);
    store_some(pm, left, m);
    store_some(pv, left, v);
    if (q.copy)
        store_some(static_cast<__bf16*>(q.copy) + e, left, w);
}

// ---------------------------------------------------------------------------
// 8-bit moments.
// ---------------------------------------------------------------------------
typedef uint8_t byte8 __attribute__((ext_vector_type(8)));
typedef uint8_t byte8a __attribute__((ext_vector_type(8), aligned(1)));

// The first n of the eight bytes at p; the others read 0 and are not touched.
__device__ __forceinline__ uint64_t load_bytes(const uint8_t* p, int64_t n)
{
    if (n >= GROUP)
        return __builtin_bit_cast(uint64_t, static_cast<byte8>(*reinterpret_cast<const byte8a*>(p)));
    uint64_t c = 0;
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        c |= static_cast<uint64_t>(i < n ? p[i] : 0) << (8 * i);
    return c;
}

__device__ __forceinline__ void store_bytes(uint8_t* p, int64_t n, uint64_t c)
{
    if (n >= GROUP) {
        *reinterpret_cast<byte8a*>(p) = __builtin_bit_cast(byte8, c);
        return;
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        if (i < n)
            p[i] = static_cast<uint8_t>(c >> (8 * i));
}

// M: the moment m (a sign and seven bits) or v (eight bits).
template <bool M>
struct Code {
    static constexpr uint32_t TOP = M ? 127 : 255, LEAST = M ? 16 : 32, BROKEN = 255;

    // The value of code c in a block with exponent byte e.
    static __device__ __forceinline__ float value(uint32_t c, uint32_t e)
    {
        const uint32_t k = c & TOP;
        uint32_t bits = k ? ((e + 1) << 23) + (k << 20) - (TOP << 20) : 0;
        if (M)
            bits |= (c & 128) << 24;
        return __uint_as_float(e == BROKEN ? 0x7fc00000u : bits);
    }

    // The exponent byte of a block whose largest magnitude has these fp32 bits.
    static __device__ __forceinline__ uint32_t exponent(uint32_t most)
    {
        const uint32_t e = most >> 23;
        return e > LEAST ? e : LEAST;
    }

    // The code of a value whose magnitude, cut to fp32 (0 below 2^-126), has these
    // bits; r: its 16 random bits.  Cutting loses nothing: r counts in units of
    // 2^-16 of a code's distance, the bits cut off lie below 2^-20 of it.
    static __device__ __forceinline__ uint32_t of(uint32_t bits, uint32_t r, uint32_t e)
    {
        if (e == BROKEN || bits == 0)
            return 0;
        const int32_t k = static_cast<int32_t>((bits + (r << 4)) >> 20) - static_cast<int32_t>((e + 1) << 3) +
                          static_cast<int32_t>(TOP);
        return static_cast<uint32_t>(k > (M ? 0 : 1) ? k : (M ? 0 : 1));
    }
};

// The fp32 bits of |x| cut by dropping bits: 0 below 2^-126, at least
// infinity's past fp32's range and for NaN.
__device__ __forceinline__ uint32_t cut(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x) & 0x7fffffffe0000000ull;
    const float f = static_cast<float>(__builtin_bit_cast(double, b));
    return b < (uint64_t(1023 - 126) << 52) ? 0 : __float_as_uint(f) & 0x7fffffffu;
}

// The largest of the 16 lanes that hold a block.
__device__ __forceinline__ uint32_t block_max(uint32_t v)
{
#pragma unroll
    for (int d = 1; d < ADAMW_BLOCK / GROUP; d <<= 1) {
        const uint32_t o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void step_coded_kernel(const AdamwGroup a, Rates r)
{
    const double scale = r.scale ? *r.scale : 1.f;
    if (!isfinite(scale))
        return;
    read_clock(r);
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const int64_t e = static_cast<int64_t>(blockIdx.x - a.first_block[t]) * ADAMW_CHUNK + threadIdx.x * GROUP;
    // Past the tensor's end: a thread works on zeros and stores nothing, so that
    // the lanes of a block stay together.
    const int64_t left = q.n - e, block = e / ADAMW_BLOCK;
    uint8_t* pm = static_cast<uint8_t*>(q.m) + e;
    uint8_t* pv = static_cast<uint8_t*>(q.v) + e;
    double s[GROUP] = {};
    float w[GROUP] = {};
    uint64_t cm = 0, cv = 0;
    uint32_t em = 0, ev = 0;
    if (left > 0) {
        load_some(q.W + e, left, w);
        cm = load_bytes(pm, left);
        cv = load_bytes(pv, left);
        em = q.exponents[2 * block];
        ev = q.exponents[2 * block + 1];
        sum_workers(static_cast<const T*>(q.G) + e, q.stride, q.P, left, s);
    }
    const float decay = static_cast<float>(r.lr * q.weight_decay);
    uint32_t am[GROUP], av[GROUP], most_m = 0, most_v = 0, minus = 0;
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const double g = s[i] * scale;
        const double m0 = Code<true>::value((cm >> (8 * i)) & 255, em), v0 = Code<false>::value((cv >> (8 * i)) & 255, ev);
        const double m = r.beta1 * m0 + r.one_beta1 * g;
        const double v = r.beta2 * v0 + r.one_beta2 * (g * g);
        w[i] = stepped(w[i], static_cast<float>(m), static_cast<float>(v), decay, r);
        am[i] = cut(m);
        av[i] = cut(v);
        minus |= static_cast<uint32_t>(__builtin_bit_cast(uint64_t, m) >> 63) << i;
        most_m = am[i] > most_m ? am[i] : most_m;
        most_v = av[i] > most_v ? av[i] : most_v;
    }
    em = Code<true>::exponent(block_max(most_m));
    ev = Code<false>::exponent(block_max(most_v));
    if (left <= 0)
        return;
    uint32_t bits[4] = {0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    if (r.rng)
        philox(Rng{static_cast<uint64_t>(r.rng[0]), static_cast<uint64_t>(r.rng[1])},
               static_cast<uint64_t>(q.first_group + e / GROUP), bits);
    cm = cv = 0;
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const uint32_t u = i & 1 ? bits[i >> 1] >> 16 : bits[i >> 1] & 0xffffu;
        const uint32_t uv = r.rng ? (u & 255) << 8 | u >> 8 : u;
        cm |= static_cast<uint64_t>(Code<true>::of(am[i], u, em) | (minus >> i & 1) << 7) << (8 * i);
        cv |= static_cast<uint64_t>(Code<false>::of(av[i], uv, ev)) << (8 * i);
    }
    store_some(q.W + e, left, w);
    store_bytes(pm, left, cm);
    store_bytes(pv, left, cv);
    if (e % ADAMW_BLOCK == 0) {
        q.exponents[2 * block] = static_cast<uint8_t>(em);
        q.exponents[2 * block + 1] = static_cast<uint8_t>(ev);
    }
    if (q.copy)
        store_some(static_cast<__bf16*>(q.copy) + e, left, w);
}

// The moments as fp32: to W (m) and copy (v) of the item, where not NULL.
__global__ __launch_bounds__(THREADS) void values_kernel(const AdamwGroup a)
{
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const int64_t e = static_cast<int64_t>(blockIdx.x - a.first_block[t]) * ADAMW_CHUNK + threadIdx.x * GROUP;
    const int64_t left = q.n - e, block = e / ADAMW_BLOCK;
    if (left <= 0)
        return;
    float x[GROUP];
    float* out = static_cast<float*>(q.copy);
    if (!q.exponents) {
        if (q.W) {
            load_some(static_cast<const float*>(q.m) + e, left, x);
            store_some(q.W + e, left, x);
        }
        if (out) {
            load_some(static_cast<const float*>(q.v) + e, left, x);
            store_some(out + e, left, x);
        }
        return;
    }
    const uint32_t em = q.exponents[2 * block], ev = q.exponents[2 * block + 1];
    if (q.W) {
        const uint64_t c = load_bytes(static_cast<const uint8_t*>(q.m) + e, left);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            x[i] = Code<true>::value((c >> (8 * i)) & 255, em);
        store_some(q.W + e, left, x);
    }
    if (out) {
        const uint64_t c = load_bytes(static_cast<const uint8_t*>(q.v) + e, left);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            x[i] = Code<false>::value((c >> (8 * i)) & 255, ev);
        store_some(out + e, left, x);
    }
}

// ---------------------------------------------------------------------------
// The gradients' norm: each workgroup's sum of squares, then their sum, both in
// a fixed order.
// ---------------------------------------------------------------------------
__device__ __forceinline__ double workgroup_sum(double v)
{
    __shared__ double lds[THREADS / 64];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i)
        v += lds[i];
    return v;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void squares_kernel(const AdamwGroup a, int64_t chunk,
                                                          double* __restrict__ partial)
{
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const int64_t first = static_cast<int64_t>(blockIdx.x - a.first_block[t]) * chunk;
    const int64_t end = first + chunk < q.n ? first + chunk : q.n;
    double sum = 0.0;
    for (int64_t e = first + threadIdx.x * GROUP; e < end; e += THREADS * GROUP) {
        double s[GROUP];
        sum_workers(static_cast<const T*>(q.G) + e, q.stride, q.P, end - e, s);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            sum = fma(s[i], s[i], sum);
        if (q.copy) {
            float x[GROUP];
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                x[i] = static_cast<float>(s[i]);
            store_some(static_cast<float*>(q.copy) + e, end - e, x);
        }
    }
    sum = workgroup_sum(sum);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(THREADS) void norm_kernel(const double* __restrict__ partial, int64_t parts,
                                                       double max_norm, float* __restrict__ result)
{
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < parts; i += THREADS)
        sum += partial[i];
    sum = workgroup_sum(sum);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        result[0] = static_cast<float>(norm);
        result[1] = !isfinite(norm) ? NAN : norm > max_norm ? static_cast<float>(max_norm / norm) : 1.f;
    }
}

}  // namespace

hipError_t launch_adamw_step(const AdamwGroup& group, int32_t dtype, bool coded, const poseidon_adamw_rule& rule,
                             hipStream_t stream)
{
    Rates r{};
    r.beta1 = rule.beta1;
    r.beta2 = rule.beta2;
    r.one_beta1 = 1.0 - rule.beta1;
    r.one_beta2 = 1.0 - rule.beta2;
    r.lr = rule.lr;
    r.eps = static_cast<float>(rule.eps);
    r.clock = rule.clock;
    r.scale = rule.scale;
    r.rng = rule.rng;
    if (!rule.clock) {
        const double t = static_cast<double>(rule.step);
        r.rate = static_cast<float>(rule.lr / (1.0 - pow(rule.beta1, t)));
        r.root = static_cast<float>(1.0 / sqrt(1.0 - pow(rule.beta2, t)));
    }
    const bool bf16 = dtype == POSEIDON_BF16;
    auto* k = coded ? (bf16 ? step_coded_kernel<__bf16> : step_coded_kernel<float>)
                    : (bf16 ? step_kernel<__bf16> : step_kernel<float>);
    k<<<group.blocks, THREADS, 0, stream>>>(group, r);
    return hipGetLastError();
}

hipError_t launch_adamw_values(const AdamwGroup& group, hipStream_t stream)
{
    values_kernel<<<group.blocks, THREADS, 0, stream>>>(group);
    return hipGetLastError();
}

hipError_t launch_adamw_squares(const AdamwGroup& group, int32_t dtype, int64_t chunk, double* partial,
                                hipStream_t stream)
{
    auto* k = dtype == POSEIDON_BF16 ? squares_kernel<__bf16> : squares_kernel<float>;
    k<<<group.blocks, THREADS, 0, stream>>>(group, chunk, partial);
    return hipGetLastError();
}

hipError_t launch_adamw_norm(const double* partial, int64_t parts, double max_norm, float* result, hipStream_t stream)
{
    norm_kernel<<<1, THREADS, 0, stream>>>(partial, parts, max_norm, result);
    return hipGetLastError();
}

}  // namespace poseidon
