// AdamW over many tensors, the gradients' norm, and the values of 8-bit moments
// (include/poseidon.h gives the formulas and the code's layout).  All of it is a few
// operations per value (77 with 8-bit moments), bound by memory: every array is read
// once and written once.  VGG19-22K's 229M values with a bf16 copy: one fp32 row of
// gradients and fp32 moments 1.23 ms (5.6 TB/s; a device copy reaches 4.8), a bf16 row
// and 8-bit moments 0.65 ms (5.7 TB/s, vector units 0.8 busy), their values 0.41 ms;
// the norm 0.14 ms (6.6 TB/s).
//
// The tensors' descriptors travel by value in the kernel arguments; a workgroup finds
// its tensor by counting the first blocks that it has reached, and works on `chunk`
// values of it, eight a thread and turn; only a tensor's last turn asks how many of
// them there are.
#include <math.h>

#include "elements.h"
#include "optimizer.h"

namespace poseidon {
namespace {

constexpr int THREADS = 256;
static_assert(ADAMW_CHUNK == THREADS * GROUP, "one group a thread");

// The tensor of workgroup b: the number of later tensors whose first block it has
// reached, eight by eight (independent scalar loads instead of a search's chain of
// them).
__device__ __forceinline__ int tensor_of(const AdamwGroup& a, int b)
{
    int t = 0;
    for (int k = 0; k < a.count; k += 8) {
        int here = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)   // (past the last tensor: first blocks beyond any)
            here += a.first_block[k + i] <= b ? 1 : 0;
        t += here;
        if (here < 8)
            break;
    }
    return t - 1;
}

// ---------------------------------------------------------------------------
// fp32 arrays go four values a thread, so that a wave's access is of 1 KB in a row;
// a turn's 2048 values are two such quads a thread, QUAD_GAP apart.  Each value is
// read and written once: past the caches.  (VGG19-22K, fp32 moments: 1.23 ms so, 1.31
// with eight neighbours a thread, 1.30 with cached loads.)
// ---------------------------------------------------------------------------
constexpr int QUAD = 4;
constexpr int QUAD_GAP = THREADS * QUAD;

typedef __bf16 bf4e __attribute__((ext_vector_type(4)));
typedef __bf16 bf4a __attribute__((ext_vector_type(4), aligned(2)));

// The quad at p: whole, or (FULL = false) the first `left` of it, the others 0.
template <bool FULL>
__device__ __forceinline__ f4e get(const float* p, int64_t left)
{
    if (FULL || left >= QUAD)
        return __builtin_nontemporal_load(reinterpret_cast<const f4a*>(p));
    f4e v;
#pragma unroll
    for (int i = 0; i < QUAD; ++i)
        v[i] = i < left ? p[i] : 0.f;
    return v;
}

template <bool FULL>
__device__ __forceinline__ bf4e get(const __bf16* p, int64_t left)
{
    if (FULL || left >= QUAD)
        return __builtin_nontemporal_load(reinterpret_cast<const bf4a*>(p));
    bf4e v;
#pragma unroll
    for (int i = 0; i < QUAD; ++i)
        v[i] = i < left ? p[i] : static_cast<__bf16>(0.f);
    return v;
}

template <bool FULL>
__device__ __forceinline__ void put(float* p, int64_t left, f4e v)
{
    if (FULL || left >= QUAD) {
        __builtin_nontemporal_store(v, reinterpret_cast<f4a*>(p));
        return;
    }
#pragma unroll
    for (int i = 0; i < QUAD; ++i)
        if (i < left)
            p[i] = v[i];
}

template <bool FULL>
__device__ __forceinline__ void put(__bf16* p, int64_t left, f4e v)
{
    const bf4e r = __builtin_convertvector(v, bf4e);
    if (FULL || left >= QUAD) {
        __builtin_nontemporal_store(r, reinterpret_cast<bf4a*>(p));
        return;
    }
#pragma unroll
    for (int i = 0; i < QUAD; ++i)
        if (i < left)
            p[i] = r[i];
}

// Adds N workers' values to s, in the workers' order, all in flight together.
template <int N, bool FULL, typename T>
__device__ __forceinline__ void add_workers(const T* g, int64_t stride, int64_t left, double (&s)[2][QUAD])
{
    decltype(get<FULL>(g, left)) r[N][2];
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            r[c][k] = get<FULL>(g + c * stride + k * QUAD_GAP, left - k * QUAD_GAP);
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < QUAD; ++i)
                s[k][i] += static_cast<float>(r[c][k][i]);
}

// The same for eight neighbours (8-bit moments): 16 bytes of bf16 past the caches; the
// two halves of fp32's 32 meet there.
__device__ __forceinline__ void get_group(const __bf16* p, Raw<__bf16>& r)
{
    r.v = __builtin_nontemporal_load(reinterpret_cast<const bf8a*>(p));
}
__device__ __forceinline__ void get_group(const float* p, Raw<float>& r) { load_raw(p, GROUP, r); }

template <int N, bool FULL, typename T>
__device__ __forceinline__ void add_workers(const T* g, int64_t stride, int64_t left, double (&s)[GROUP])
{
    Raw<T> r[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        if constexpr (FULL)
            get_group(g + c * stride, r[c]);
        else
            load_raw(g + c * stride, left, r[c]);
    }
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            s[i] += raw_value(r[c], i);
}

// Sum over the workers, in 64 bits and in the workers' order, MOST of them in flight.
template <int MOST, bool FULL, typename T, typename S>
__device__ __forceinline__ void sum_workers(const T* g, int64_t stride, int P, int64_t left, S& s)
{
    for (; P >= MOST; P -= MOST, g += MOST * stride)
        add_workers<MOST, FULL>(g, stride, left, s);
    if (MOST > 4 && P & 4) {
        add_workers<4, FULL>(g, stride, left, s);
        g += 4 * stride;
    }
    if (P & 2) {
        add_workers<2, FULL>(g, stride, left, s);
        g += 2 * stride;
    }
    if (P & 1)
        add_workers<1, FULL>(g, stride, left, s);
}

// b^t for t >= 1, by squaring: each squaring doubles the relative error and adds a
// rounding, so it is within about t b^t 2^-53 of it, which is below 2^-54 / (1 - b) (2^-41
// at 0.9999, 2^-31 at 0.9999999) and, of 1 - b^t, below 2^-53 / (1 - b): less than a
// rounding to fp32 up to b = 1 - 2^-29.
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
    float b1, b1_rest, b2, b2_rest;   // the betas in two parts (part_of)
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

// W - lr (decay W + (m / c1) / (sqrt(v / c2) + eps)).  The square root and the
// reciprocal are the instructions' (1 ulp each) unless CAREFUL (needs_care).
template <bool CAREFUL>
__device__ __forceinline__ float stepped(float w, float m, float v, float decay, const Rates& r)
{
    if (CAREFUL)
        return w - fmaf(decay, w, r.rate * m / fmaf(sqrtf(v), r.root, r.eps));
    return w - fmaf(decay, w, r.rate * m * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v), r.root, r.eps)));
}

// The values of a workgroup of item q: from `first` up to `end`, in turns.
struct Range {
    int64_t first, end;
};

__device__ __forceinline__ Range range_of(const AdamwItem& q, int64_t block, int64_t chunk)
{
    const int64_t first = block * chunk;
    return Range{first, first + chunk < q.n ? first + chunk : q.n};
}

// f(full, at) for its turns, full: of whole groups throughout the workgroup.
template <typename F>
__device__ __forceinline__ void turns(const Range& r, F&& f)
{
    int64_t at = r.first;
    for (; at + ADAMW_CHUNK <= r.end; at += ADAMW_CHUNK)
        f(std::true_type(), at);
    if (at < r.end)
        f(std::false_type(), at);
}

// ---------------------------------------------------------------------------
// The step with fp32 moments.  ONE: one worker's rows, or their sums; its product
// with the scale rounds alike in 32 and 64 bits.  A beta is taken in two parts: rounded
// to fp32 it would put every moment off by up to 2^-25 / (1 - beta) for good (1.4e-3 at
// 0.99999), since the two factors would not add up to 1.
// ---------------------------------------------------------------------------
template <typename T, bool CAREFUL, bool ONE>
__global__ __launch_bounds__(THREADS) void step_kernel(const AdamwGroup a, Rates r)
{
    const float scale = r.scale ? *r.scale : 1.f;
    if (!isfinite(scale))
        return;
    read_clock(r);
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const float o1 = static_cast<float>(r.one_beta1), o2 = static_cast<float>(r.one_beta2);
    const float decay = static_cast<float>(r.lr * q.weight_decay);
    const Range range = range_of(q, blockIdx.x - a.first_block[t], a.chunk);
    turns(range, [&](auto full, int64_t at) {
        constexpr bool FULL = decltype(full)::value;
        const int64_t e = at + threadIdx.x * QUAD, left = q.n - e;
        float* const pw = q.W + e;
        float* const pm = static_cast<float*>(q.m) + e;
        float* const pv = static_cast<float*>(q.v) + e;
        const T* const pg = static_cast<const T*>(q.G) + e;
        f4e w[2], m[2], v[2], g[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            w[k] = get<FULL>(pw + k * QUAD_GAP, left - k * QUAD_GAP);
            m[k] = get<FULL>(pm + k * QUAD_GAP, left - k * QUAD_GAP);
            v[k] = get<FULL>(pv + k * QUAD_GAP, left - k * QUAD_GAP);
        }
        if constexpr (ONE) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                g[k] = __builtin_convertvector(get<FULL>(pg + k * QUAD_GAP, left - k * QUAD_GAP), f4e) * scale;
        } else {
            double s[2][QUAD] = {};
            sum_workers<4, FULL>(pg, q.stride, q.P, left, s);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < QUAD; ++i)
                    g[k][i] = static_cast<float>(s[k][i] * scale);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int i = 0; i < QUAD; ++i) {
                m[k][i] = fmaf(r.b1, m[k][i], fmaf(r.b1_rest, m[k][i], o1 * g[k][i]));
                v[k][i] = fmaf(r.b2, v[k][i], fmaf(r.b2_rest, v[k][i], o2 * (g[k][i] * g[k][i])));
                w[k][i] = stepped<CAREFUL>(w[k][i], m[k][i], v[k][i], decay, r);
            }
            put<FULL>(pw + k * QUAD_GAP, left - k * QUAD_GAP, w[k]);
            put<FULL>(pm + k * QUAD_GAP, left - k * QUAD_GAP, m[k]);
            put<FULL>(pv + k * QUAD_GAP, left - k * QUAD_GAP, v[k]);
            if (q.copy)
                put<FULL>(static_cast<__bf16*>(q.copy) + e + k * QUAD_GAP, left - k * QUAD_GAP, w[k]);
        }
    });
}

// ---------------------------------------------------------------------------
// 8-bit moments.
// ---------------------------------------------------------------------------
typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef uint32_t word2a __attribute__((ext_vector_type(2), aligned(1)));

// Eight bytes, or the first n of them; the others read 0 and are not touched.
template <bool FULL>
__device__ __forceinline__ word2 load_bytes(const uint8_t* p, int64_t n)
{
    if (FULL || n >= GROUP)
        return __builtin_nontemporal_load(reinterpret_cast<const word2a*>(p));
    word2 c{0, 0};
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        c[i >> 2] |= static_cast<uint32_t>(i < n ? p[i] : 0) << (8 * (i & 3));
    return c;
}

template <bool FULL>
__device__ __forceinline__ void store_bytes(uint8_t* p, int64_t n, word2 c)
{
    if (FULL || n >= GROUP) {
        __builtin_nontemporal_store(c, reinterpret_cast<word2a*>(p));
        return;
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        if (i < n)
            p[i] = static_cast<uint8_t>(c[i >> 2] >> (8 * (i & 3)));
}

__device__ __forceinline__ double from_high(uint32_t high)
{
    return __builtin_bit_cast(double, static_cast<uint64_t>(high) << 32);
}

__device__ __forceinline__ uint32_t high_of(double x)
{
    return static_cast<uint32_t>(__builtin_bit_cast(uint64_t, x) >> 32);
}

// M: the moment m (a sign and seven bits) or v (eight bits).  A code's value is put
// together, and a moment's code taken, as the high word of its fp64 bits, whose
// exponent is fp32's plus 896 and where a code is bits 17 and up.
template <bool M>
struct Code {
    static constexpr uint32_t TOP = M ? 127 : 255, LEAST = M ? 16 : 32, BROKEN = 255, MORE = 1023 - 127;

    // What is added to a code's bits in a block of exponent byte e.
    static __device__ __forceinline__ uint32_t base(uint32_t e) { return ((e + 1 + MORE) << 20) - (TOP << 17); }

    // The value of byte i of the codes c.
    static __device__ __forceinline__ double value(word2 c, int i, uint32_t base)
    {
        const uint32_t w = c[i >> 2], k = w >> (8 * (i & 3)) & TOP;
        uint32_t high = k ? (k << 17) + base : 0;
        if (M)
            high |= w << (24 - 8 * (i & 3)) & 0x80000000u;
        return from_high(high);
    }

    // The exponent byte of a block whose largest magnitude has this high word.
    static __device__ __forceinline__ uint32_t exponent(uint32_t most)
    {
        const int32_t e = static_cast<int32_t>(most >> 20) - static_cast<int32_t>(MORE);
        return static_cast<uint32_t>(e < static_cast<int32_t>(LEAST) ? LEAST : e > static_cast<int32_t>(BROKEN) ? BROKEN : e);
    }

    // The code of a magnitude with high word x; r: its 16 random bits, which count in
    // 2^-16 of the distance to the next code: the low word and one bit of the high lie
    // below that and cannot carry into it.  m's magnitudes below 2^-126 end below
    // code 1 by themselves.
    static __device__ __forceinline__ uint32_t of(uint32_t x, uint32_t r, uint32_t e)
    {
        const int32_t k = static_cast<int32_t>((x + (r << 1)) >> 17) - static_cast<int32_t>(((e + 1 + MORE) << 3) - TOP);
        const int32_t most = e == BROKEN ? 0 : static_cast<int32_t>(TOP);
        if (M)
            return static_cast<uint32_t>(k < 0 ? 0 : k > most ? most : k);
        const int32_t least = e == BROKEN || x < ((1023 - 126) << 20) ? 0 : 1;
        return static_cast<uint32_t>(least == 0 ? 0 : k < 1 ? 1 : k > most ? most : k);
    }
};

// The largest of the 16 lanes (a row of the wave) that hold a block.
__device__ __forceinline__ uint32_t block_max(uint32_t v)
{
#define ROTATED(by)                                                                                                  \
    {                                                                                                                \
        const uint32_t o = static_cast<uint32_t>(                                                                    \
            __builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x120 | by, 0xf, 0xf, true));                              \
        v = o > v ? o : v;                                                                                           \
    }
    ROTATED(8)
    ROTATED(4)
    ROTATED(2)
    ROTATED(1)
#undef ROTATED
    return v;
}

// One group of eight neighbours.  Past the tensor's end (FULL = false) a thread works
// on zeros and stores nothing, so that the lanes of a block stay together.
template <typename T, bool CAREFUL, bool FULL, bool ONE>
__device__ __forceinline__ void step_coded(const AdamwItem& q, int64_t e, const Rates& r, double scale, float decay,
                                           const Rng& rng)
{
    const int64_t left = q.n - e;
    const bool any = FULL || left > 0;
    uint8_t* const pm = static_cast<uint8_t*>(q.m) + e;
    uint8_t* const pv = static_cast<uint8_t*>(q.v) + e;
    uint8_t* const px = q.exponents + 2 * (e / ADAMW_BLOCK);
    Raw<float> rw{};
    word2 cm{0, 0}, cv{0, 0};
    uint32_t em = 0, ev = 0;
    double s[GROUP] = {};
    if (any) {
        load_raw(q.W + e, FULL ? GROUP : left, rw);   // (a thread's two halves meet in the cache)
        cm = load_bytes<FULL>(pm, left);
        cv = load_bytes<FULL>(pv, left);
        em = px[0];
        ev = px[1];
        if constexpr (ONE)
            add_workers<1, FULL>(static_cast<const T*>(q.G) + e, 0, left, s);
        else
            sum_workers<4, FULL>(static_cast<const T*>(q.G) + e, q.stride, q.P, left, s);
    }
    uint32_t bits[4] = {0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    if (r.rng)
        philox(rng, static_cast<uint64_t>(q.first_group + e / GROUP), bits);
    // A block that has lost its numbers makes NaN of whatever its codes say.
    const double b1 = em == Code<true>::BROKEN ? NAN : r.beta1, b2 = ev == Code<false>::BROKEN ? NAN : r.beta2;
    const uint32_t bm = Code<true>::base(em), bv = Code<false>::base(ev);
    uint32_t xm[GROUP], xv[GROUP], most_m = 0, most_v = 0;
    float w[GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const double g = s[i] * scale;
        const double m = b1 * Code<true>::value(cm, i, bm) + r.one_beta1 * g;
        const double v = b2 * Code<false>::value(cv, i, bv) + r.one_beta2 * (g * g);
        w[i] = stepped<CAREFUL>(raw_value(rw, i), static_cast<float>(m), static_cast<float>(v), decay, r);
        xm[i] = high_of(m);
        xv[i] = high_of(v) & 0x7fffffffu;
        const uint32_t am = xm[i] & 0x7fffffffu;
        most_m = am > most_m ? am : most_m;
        most_v = xv[i] > most_v ? xv[i] : most_v;
    }
    em = Code<true>::exponent(block_max(most_m));
    ev = Code<false>::exponent(block_max(most_v));
    if (!any)
        return;
    cm = cv = word2{0, 0};
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const uint32_t u = i & 1 ? bits[i >> 1] >> 16 : bits[i >> 1] & 0xffffu;
        const uint32_t uv = r.rng ? (u & 255) << 8 | u >> 8 : u;
        const uint32_t k = Code<true>::of(xm[i] & 0x7fffffffu, u, em) | (xm[i] >> 24 & 128);
        cm[i >> 2] |= k << (8 * (i & 3));
        cv[i >> 2] |= Code<false>::of(xv[i], uv, ev) << (8 * (i & 3));
    }
    store_some(q.W + e, FULL ? GROUP : left, w);
    store_bytes<FULL>(pm, left, cm);
    store_bytes<FULL>(pv, left, cv);
    if (e % ADAMW_BLOCK == 0) {
        px[0] = static_cast<uint8_t>(em);
        px[1] = static_cast<uint8_t>(ev);
    }
    if (q.copy)
        store_some(static_cast<__bf16*>(q.copy) + e, FULL ? GROUP : left, w);
}

template <typename T, bool CAREFUL, bool ONE>
__global__ __launch_bounds__(THREADS) void step_coded_kernel(const AdamwGroup a, Rates r)
{
    const double scale = r.scale ? *r.scale : 1.f;
    if (!isfinite(scale))
        return;
    read_clock(r);
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const float decay = static_cast<float>(r.lr * q.weight_decay);
    Rng rng{0, 0};
    if (r.rng)
        rng = Rng{static_cast<uint64_t>(r.rng[0]), static_cast<uint64_t>(r.rng[1])};
    const Range range = range_of(q, blockIdx.x - a.first_block[t], a.chunk);
    turns(range, [&](auto full, int64_t at) {
        step_coded<T, CAREFUL, decltype(full)::value, ONE>(q, at + threadIdx.x * GROUP, r, scale, decay, rng);
    });
}

// The moments as fp32: to W (m) and copy (v) of the item, where not NULL.
template <bool FULL, bool M>
__device__ __forceinline__ void write_values(const AdamwItem& q, int64_t e, float* out)
{
    const void* from = M ? q.m : q.v;
    if (!out)
        return;
    f4e x[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t at = e + k * QUAD_GAP, left = q.n - at;
        if (!q.exponents) {
            x[k] = get<FULL>(static_cast<const float*>(from) + at, left);
            continue;
        }
        const uint8_t* p = static_cast<const uint8_t*>(from) + at;
        word2 c{0, 0};
        uint32_t b = 0;
        if (FULL) {
            typedef uint32_t word __attribute__((aligned(1)));
            c[0] = __builtin_nontemporal_load(reinterpret_cast<const word*>(p));
            b = q.exponents[2 * (at / ADAMW_BLOCK) + !M];
        } else if (left > 0) {
#pragma unroll
            for (int i = 0; i < QUAD; ++i)
                c[0] |= static_cast<uint32_t>(i < left ? p[i] : 0) << (8 * i);
            b = q.exponents[2 * (at / ADAMW_BLOCK) + !M];
        }
#pragma unroll
        for (int i = 0; i < QUAD; ++i)
            x[k][i] = b == Code<M>::BROKEN ? NAN : static_cast<float>(Code<M>::value(c, i, Code<M>::base(b)));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        put<FULL>(out + e + k * QUAD_GAP, q.n - e - k * QUAD_GAP, x[k]);
}

__global__ __launch_bounds__(THREADS) void values_kernel(const AdamwGroup a)
{
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const Range range = range_of(q, blockIdx.x - a.first_block[t], a.chunk);
    turns(range, [&](auto full, int64_t at) {
        const int64_t e = at + threadIdx.x * QUAD;
        write_values<decltype(full)::value, true>(q, e, q.W);
        write_values<decltype(full)::value, false>(q, e, static_cast<float*>(q.copy));
    });
}

// ---------------------------------------------------------------------------
// The gradients' norm: each workgroup's sum of squares, then their sum, both in
// a fixed order.
// ---------------------------------------------------------------------------
template <int N>
__device__ __forceinline__ double workgroup_sum(double v)
{
    __shared__ double lds[N / 64];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < N / 64; ++i)
        v += lds[i];
    return v;
}

template <typename T, bool ONE>
__global__ __launch_bounds__(THREADS) void squares_kernel(const AdamwGroup a, double* __restrict__ partial)
{
    const int t = tensor_of(a, blockIdx.x);
    const AdamwItem& q = a.item[t];
    const Range range = range_of(q, blockIdx.x - a.first_block[t], a.chunk);
    double sum = 0.0;
    float most = 0.f;   // of the sums as fp32
    turns(range, [&](auto full, int64_t at) {
        constexpr bool FULL = decltype(full)::value;
        const int64_t e = at + threadIdx.x * QUAD, left = q.n - e;
        double s[2][QUAD] = {};
        if constexpr (ONE)
            add_workers<1, FULL>(static_cast<const T*>(q.G) + e, 0, left, s);
        else   // (eight workers' fp32 values would take the registers of half of the waves)
            sum_workers<sizeof(T) == 2 ? 8 : 4, FULL>(static_cast<const T*>(q.G) + e, q.stride, q.P, left, s);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f4e x;
#pragma unroll
            for (int i = 0; i < QUAD; ++i) {
                sum = fma(s[k][i], s[k][i], sum);
                x[i] = static_cast<float>(s[k][i]);
                if (!ONE)
                    most = fmaxf(most, fabsf(x[i]));
            }
            if (q.copy)
                put<FULL>(static_cast<float*>(q.copy) + e + k * QUAD_GAP, left - k * QUAD_GAP, x);
        }
    });
    // A kept sum that is infinite in fp32 makes the norm infinite: the step from the sums
    // would be wrong, so it is left out.
    if (!ONE && q.copy && most == INFINITY)
        sum = INFINITY;
    sum = workgroup_sum<THREADS>(sum);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = sum;
}

constexpr int NORM_THREADS = 1024;

__global__ __launch_bounds__(NORM_THREADS) void norm_kernel(const double* __restrict__ partial, int64_t parts,
                                                            double max_norm, float* __restrict__ result)
{
    double sum = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < parts; i += NORM_THREADS)
        sum += partial[i];
    sum = workgroup_sum<NORM_THREADS>(sum);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        result[0] = static_cast<float>(norm);
        result[1] = !isfinite(norm) ? NAN : norm > max_norm ? static_cast<float>(max_norm / norm) : 1.f;
    }
}

}  // namespace

// The largest fp32 value below b (0 for 0): what is left of b is above 0, so that an
// infinite moment times either part is that infinity.
static float part_of(double b)
{
    const float f = static_cast<float>(b);
    return f < b || f == 0.f ? f : nextafterf(f, 0.f);
}

// The instructions take denormals for 0.  Of a v below 2^-126 the denominator then lacks
// up to 2^-63 root, root = (1 - beta2^t)^-1/2 <= (1 - beta2)^-1/2: less than a rounding of
// eps where that is 2^24 times as large.  And the reciprocal is 0 above 2^126, which only
// eps can bring about (v's root ends at 2^64, root at 2^27).
static bool needs_care(const Rates& r)
{
    return !(r.eps >= 0x1p-39 / sqrt(r.one_beta2) && r.eps < 0x1p125f);
}

hipError_t launch_adamw_step(const AdamwGroup& group, int32_t dtype, AdamwKind kind, const poseidon_adamw_rule& rule,
                             hipStream_t stream)
{
    Rates r{};
    r.beta1 = rule.beta1;
    r.beta2 = rule.beta2;
    r.one_beta1 = 1.0 - rule.beta1;
    r.one_beta2 = 1.0 - rule.beta2;
    r.b1 = part_of(rule.beta1);
    r.b1_rest = static_cast<float>(rule.beta1 - r.b1);
    r.b2 = part_of(rule.beta2);
    r.b2_rest = static_cast<float>(rule.beta2 - r.b2);
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
    auto pick = [&](auto careful, auto one) {
        constexpr bool CAREFUL = decltype(careful)::value, ONE = decltype(one)::value;
        if (dtype == POSEIDON_BF16)
            return kind.coded ? step_coded_kernel<__bf16, CAREFUL, ONE> : step_kernel<__bf16, CAREFUL, ONE>;
        return kind.coded ? step_coded_kernel<float, CAREFUL, ONE> : step_kernel<float, CAREFUL, ONE>;
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    auto* k = needs_care(r) ? (kind.one ? pick(yes, yes) : pick(yes, no)) : (kind.one ? pick(no, yes) : pick(no, no));
    k<<<group.blocks, THREADS, 0, stream>>>(group, r);
    return hipGetLastError();
}

hipError_t launch_adamw_values(const AdamwGroup& group, hipStream_t stream)
{
    values_kernel<<<group.blocks, THREADS, 0, stream>>>(group);
    return hipGetLastError();
}

hipError_t launch_adamw_squares(const AdamwGroup& group, int32_t dtype, bool one, double* partial, hipStream_t stream)
{
    auto* k = dtype == POSEIDON_BF16 ? (one ? squares_kernel<__bf16, true> : squares_kernel<__bf16, false>)
                                     : (one ? squares_kernel<float, true> : squares_kernel<float, false>);
    k<<<group.blocks, THREADS, 0, stream>>>(group, partial);
    return hipGetLastError();
}

hipError_t launch_adamw_norm(const double* partial, int64_t parts, double max_norm, float* result, hipStream_t stream)
{
    norm_kernel<<<1, NORM_THREADS, 0, stream>>>(partial, parts, max_norm, result);
    return hipGetLastError();
}

}  // namespace poseidon
