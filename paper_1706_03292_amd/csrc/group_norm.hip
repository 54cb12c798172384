// Group norm with an activation, channels last, and its backward pass
// (include/poseidon.h gives the formulas).  A few operations per value, bound by
// memory: x (and dy) read, y (dx) written once each is what it cannot do without.
// bf16: forward 32 x 56 x 56 x 256 in one launch 30 us (3.4 TB/s of that), 32 x 224 x
// 224 x 64 in two 113 us (3.6: x is read twice), backward 32 x 56 x 56 x 256 in
// three 55 us (2.8).
//
// A sample is L rows of C channels.  Threads stand in teams of a row each, a thread
// at eight neighbouring channels (a column), and walk the rows.  Maps whose groups
// fit a workgroup's registers are read once (held_*_kernel).  Others take three
// launches: sums of each chunk of rows and channel; each group's statistics from
// them (two launches for wide groups); the result, from a second read.  Where the
// chunks are few, the first launch sums up groups too and the last one joins them: two.
//
// A row that does not divide into eights has its last column end with it: that
// thread's first `skip` channels belong to the column before, count for no sum and
// are stored twice, alike.  So every access is of eight values (fewer channels than
// eight in all are read one by one).
//
// Sums over a thread's rows and a workgroup's teams are fp32 (a held group's over its
// channels too), what joins chunks, and channels elsewhere, is in 64 bits.  Forward,
// they are sums of differences from a value of the group or from a first mean, and the
// result counts with what the mean's rounding to fp32 leaves (as part of beta), so that
// a mean far from 0 costs y no accuracy.  The backward pass takes the mean as it is
// handed over.  Every order is fixed: nothing depends on timing.
#include "elements.h"

namespace poseidon {
namespace {

constexpr int SUM_THREADS = 256;

__host__ __device__ __forceinline__ int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A pair of sums.
struct Pair {
    float a, b;
};

// The map, and how it is cut: workgroups of `teams` rows of `cols` columns, `sides`
// of them across a row; `chunks` of `rows` rows down a sample.
struct Map {
    int64_t N, L, C, groups, rows, chunks, work;   // work: workgroups
    int32_t D, cols, sides, teams, threads;        // D: channels a group
    int32_t piece;     // channels of one group that lie together in every thread's eight
    int32_t shift;     // its logarithm
    int32_t fold;      // cols is a power of two up to 64: a wave's teams are joined by shuffles
    int32_t span;      // groups of a workgroup (held)
    int32_t lanes;     // that add up one group (held, chunk): a power of two up to 64
    int32_t slices;    // threads that add up one group's chunks
    float inv_D;
};

// channel / D, for channels below 2^16: the quotient's distance from the next
// integer is at least 1 / (2 D), its error below 2^-22 of it.
__device__ __forceinline__ int group_of(const Map& h, int channel)
{
    return static_cast<int>((static_cast<float>(channel) + 0.5f) * h.inv_D);
}

// Where a thread stands.
struct Spot {
    int64_t n, first_row, end_row;   // of its sample; rows of its chunk
    int64_t base;                    // of its first row's first value
    int channel, first;              // its first channel, its workgroup's first channel
    int col, team, skip;
    bool active;
};

__device__ __forceinline__ Spot spot_of(const Map& h, int64_t b)
{
    Spot s;
    const int side = static_cast<int>(b % h.sides);
    b /= h.sides;
    s.n = b / h.chunks;
    s.first_row = (b - s.n * h.chunks) * h.rows;
    s.end_row = s.first_row + h.rows < h.L ? s.first_row + h.rows : h.L;
    s.col = static_cast<int>(threadIdx.x) % h.cols;
    s.team = static_cast<int>(threadIdx.x) / h.cols;
    const int C = static_cast<int>(h.C), at = (side * h.cols + s.col) * GROUP;
    s.first = side * h.cols * GROUP;
    s.active = s.team < h.teams && at < C;
    s.channel = at + GROUP <= C || C < GROUP ? at : C - GROUP;
    s.skip = at - s.channel;
    s.base = (s.n * h.L + s.first_row + s.team) * h.C + s.channel;
    return s;
}

// Eight values of a row, or all of a row of fewer.
template <typename T>
__device__ __forceinline__ void load_row(const Map& h, const T* p, Raw<T>& r)
{
    if (h.C >= GROUP)
        load_raw(p, GROUP, r);
    else
        load_raw(p, h.C, r);
}

template <typename T>
__device__ __forceinline__ void store_row(const Map& h, T* p, const float (&v)[GROUP])
{
    if (h.C >= GROUP)
        store_group(p, v);
    else
        store_some(p, h.C, v);
}

template <typename T>
__device__ __forceinline__ void values_of(const Raw<T>& r, float (&v)[GROUP])
{
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        v[i] = raw_value(r, i);
}

// The same for a result that is not read again here, past the caches: what the second
// read of a large map finds there stays (32 x 224 x 224 x 64 bf16, forward 137 us with
// plain stores, 117 so).
__device__ __forceinline__ void stream_group(float* p, const float (&v)[GROUP])
{
    f4a a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = v[i];
        b[i] = v[4 + i];
    }
    __builtin_nontemporal_store(a, reinterpret_cast<f4a*>(p));
    __builtin_nontemporal_store(b, reinterpret_cast<f4a*>(p + 4));
}

__device__ __forceinline__ void stream_group(__bf16* p, const float (&v)[GROUP])
{
    f8e a;
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        a[i] = v[i];
    __builtin_nontemporal_store(__builtin_convertvector(a, bf8e), reinterpret_cast<bf8a*>(p));
}

template <typename T>
__device__ __forceinline__ void stream_row(const Map& h, T* p, const float (&v)[GROUP])
{
    if (h.C >= GROUP)
        stream_group(p, v);
    else
        store_some(p, h.C, v);
}

// A weight array's values at a thread's channels.
__device__ __forceinline__ void load_weights(const Map& h, const Spot& s, const float* p, float (&v)[GROUP])
{
    load_some(p + s.channel, s.active ? h.C - s.channel : 0, v);
}

// ---------------------------------------------------------------------------
// The activation and its slope.
// ---------------------------------------------------------------------------
// 1 / (1 + e^-z), the exponential and the reciprocal by the instructions that are
// right to 1 ulp: z's product with log2 e adds |z| 2^-23 to the exponential's error.
__device__ __forceinline__ float sigmoid(float z)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

template <int ACT>
__device__ __forceinline__ float activated(float z)
{
    if (ACT == POSEIDON_ACT_RELU)
        return z > 0.f || z != z ? z : 0.f;
    if (ACT == POSEIDON_ACT_SILU)
        return z * sigmoid(z);
    return z;
}

// What a backward pass reads of its inputs besides x and dy.
struct Inputs {
    const float* gamma;
    const float* beta;
    const float* mean;
    const float* rstd;
};

// A thread's channels in the backward pass: d = x - mean, z = d scale + shift.
struct Lines {
    float mean[GROUP], scale[GROUP], shift[GROUP];
};

__device__ __forceinline__ void load_lines(const Map& h, const Spot& s, const Inputs& in, Lines& l,
                                           float (&rstd)[GROUP])
{
    load_weights(h, s, in.gamma, l.scale);
    load_weights(h, s, in.beta, l.shift);
    if (!s.active)
        return;
    const float* const mean = in.mean + s.n * h.groups;
    const float* const rstd_of = in.rstd + s.n * h.groups;
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const int c = s.channel + i < h.C ? s.channel + i : static_cast<int>(h.C) - 1, g = group_of(h, c);
        l.mean[i] = mean[g];
        rstd[i] = rstd_of[g];
        l.scale[i] *= rstd[i];
    }
}

// dz = dy act'(z) of a thread's channels, v: x, d: x - mean.
//
// ReLU: z is within 4 u (|d scale| + |shift|) of its value, u = 2^-24.  Its sign can
// be wrong only where |z| is below that, where |d scale| is |shift| but for as much:
// z below 2^-19 |shift| is made again in 64 bits, so that the side it falls on does
// not depend on how it was rounded.
template <int ACT>
__device__ __forceinline__ void slopes(const Map& h, const Spot& s, const Inputs& in, const Lines& l,
                                       const float (&v)[GROUP], const float (&d)[GROUP], float (&dz)[GROUP])
{
    if (ACT == POSEIDON_ACT_NONE)
        return;
    if (ACT == POSEIDON_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            const float z = fmaf(d[i], l.scale[i], l.shift[i]), q = sigmoid(z);
            dz[i] = dz[i] * q * fmaf(z, 1.f - q, 1.f);
        }
        return;
    }
    uint32_t on = 0, near = 0;
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const float z = fmaf(d[i], l.scale[i], l.shift[i]);
        on |= (z > 0.f ? 1u : 0u) << i;
        near |= (fabsf(z) <= fabsf(l.shift[i]) * 0x1p-19f ? 1u : 0u) << i;
    }
    for (; near; near &= near - 1) {   // (one after another: rare, and few registers)
        const int i = __builtin_ctz(near);
        float x = v[0];
#pragma unroll
        for (int k = 1; k < GROUP; ++k)
            x = i == k ? v[k] : x;
        const int c = s.channel + i < h.C ? s.channel + i : static_cast<int>(h.C) - 1;
        const int64_t g = s.n * h.groups + group_of(h, c);
        const double z = (static_cast<double>(x) - in.mean[g]) * in.rstd[g] * in.gamma[c] + in.beta[c];
        on = (on & ~(1u << i)) | (z > 0.0 ? 1u : 0u) << i;
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        dz[i] = on >> i & 1 ? dz[i] : 0.f;
}

// ---------------------------------------------------------------------------
// Maps held in registers: one workgroup takes whole groups of one sample, reads
// them once, and has all their values when it knows their statistics.  Thread
// (team, col) holds rows team, team + teams, ...: up to K of them.
// ---------------------------------------------------------------------------
constexpr int XCDS = 8;

// Neighbouring workgroups run on different dies, each with a cache of its own: the
// workgroups of one sample, which share memory lines, are given to one die.
__device__ __forceinline__ int64_t on_one_die(int64_t work)
{
    const int64_t each = gridDim.x / XCDS;
    const int64_t b = static_cast<int64_t>(blockIdx.x % XCDS) * each + blockIdx.x / XCDS;
    return b < work ? b : -1;
}

template <typename T, int K>
__device__ __forceinline__ void hold(const T* x, const Map& h, const Spot& s, Raw<T> (&r)[K])
{
    const int64_t step = h.teams * h.C;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        r[j] = Raw<T>{};
        if (s.active && s.team + j * h.teams < h.L)
            load_row(h, x + s.base + j * step, r[j]);
    }
}

// Keeps the compiler from carrying what it unpacked in one pass over the held
// values to the next, which would take twice the registers of bf16 values.
__device__ __forceinline__ void unpack_again(Raw<__bf16>& r)
{
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    u4 w = __builtin_bit_cast(u4, r);
    asm volatile("" : "+v"(w));
    r = __builtin_bit_cast(Raw<__bf16>, w);
}
__device__ __forceinline__ void unpack_again(Raw<float>&) {}

// V sums a channel (v: of this thread's rows; 0 in its skipped channels) joined over
// the workgroup's groups: out[g * V + i], in LDS.
template <int NT, int V>
__device__ __forceinline__ void join_groups(float (&v)[V][GROUP], const Map& h, const Spot& s, float* parts, float* out)
{
    const int pieces = GROUP / h.piece, skip = s.skip / h.piece;   // (piece divides 8 and the row's rest: whole pieces)
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (h.piece >= 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[i][k] = v[i][2 * k] + v[i][2 * k + 1];
        }
        if (h.piece >= 4) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                v[i][k] = v[i][2 * k] + v[i][2 * k + 1];
        }
        if (h.piece >= 8)
            v[i][0] += v[i][1];
    }
    const int each = h.D / h.piece, rows = h.fold ? NT / 64 : h.teams;   // pieces of a group and row
    int row = s.team;
    bool writes = s.active;
    if (h.fold) {
        for (int m = h.cols; m < 64; m <<= 1)
#pragma unroll
            for (int k = 0; k < GROUP; ++k)
                if (k < pieces)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        v[i][k] += __shfl_xor(v[i][k], m);
        row = threadIdx.x >> 6;
        writes = s.active && (threadIdx.x & 63) < h.cols;
    }
    __syncthreads();   // what an earlier sum left has been read
    if (writes) {
#pragma unroll
        for (int k = 0; k < GROUP; ++k)
            if (k >= skip && k < pieces) {
                const int c = s.channel - s.first + k * h.piece, g = group_of(h, c);
                if (g < h.span) {   // (past the last channel: none)
                    const int at = (g * rows + row) * each + ((c - g * h.D) >> h.shift);
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        parts[at * V + i] = v[i][k];
                }
            }
    }
    __syncthreads();
    for (int g = static_cast<int>(threadIdx.x) / h.lanes; g < h.span; g += NT / h.lanes) {
        float a[V] = {};
        const float* of = parts + g * rows * each * V;
#pragma unroll 4
        for (int q = threadIdx.x & (h.lanes - 1); q < rows * each; q += h.lanes)
#pragma unroll
            for (int i = 0; i < V; ++i)
                a[i] += of[q * V + i];
        for (int m = 1; m < h.lanes; m <<= 1)
#pragma unroll
            for (int i = 0; i < V; ++i)
                a[i] += __shfl_xor(a[i], m);
        if ((threadIdx.x & (h.lanes - 1)) == 0)
#pragma unroll
            for (int i = 0; i < V; ++i)
                out[g * V + i] = a[i];
    }
    __syncthreads();
}

// The mean is a first sum, corrected by the sum of the differences from it, which
// also gives the spread.
template <typename T, int ACT, int NT, int K>
__global__ __launch_bounds__(NT) void held_forward_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                          const float* __restrict__ beta, Map h, float eps,
                                                          T* __restrict__ y, float* __restrict__ mean_out,
                                                          float* __restrict__ rstd_out)
{
    extern __shared__ float lds[];
    const int64_t b = on_one_die(h.work);
    if (b < 0)
        return;
    const Spot s = spot_of(h, b);
    float* const sums = lds;                  // of the groups
    float* const parts = lds + 2 * h.span;
    Raw<T> r[K];
    hold(x, h, s, r);
    const float inv = 1.f / (static_cast<float>(h.L) * static_cast<float>(h.D));
    const int local = s.channel - s.first, most = h.span - 1;
    float mean[GROUP], a[1][GROUP] = {};
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            a[0][i] += raw_value(r[j], i);
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        a[0][i] = i < s.skip ? 0.f : a[0][i];
    join_groups<NT, 1>(a, h, s, parts, sums);
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const int g = group_of(h, local + i);
        mean[i] = sums[g < most ? g : most] * inv;   // (past the last channel: nothing is stored)
    }
    float c[2][GROUP] = {};
#pragma unroll
    for (int j = 0; j < K; ++j) {
        unpack_again(r[j]);
        if (s.active && s.team + j * h.teams < h.L) {
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const float d = raw_value(r[j], i) - mean[i];
                c[0][i] += d;
                c[1][i] = fmaf(d, d, c[1][i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        const bool own = i >= s.skip && s.channel + i < h.C;
        c[0][i] = own ? c[0][i] : 0.f;
        c[1][i] = own ? c[1][i] : 0.f;
    }
    float scale[GROUP], shift[GROUP];
    load_weights(h, s, gamma, scale);
    load_weights(h, s, beta, shift);
    join_groups<NT, 2>(c, h, s, parts, sums);
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        int g = group_of(h, local + i);
        g = g < most ? g : most;
        const float off = sums[2 * g] * inv, var = sums[2 * g + 1] * inv - off * off;
        const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);   // (NaN stays)
        // the mean rounded to fp32, and what that leaves of it (the exact error of the sum)
        const float sum = mean[i] + off, part = sum - mean[i];
        const float low = (mean[i] - (sum - part)) + (off - part);
        mean[i] = sum;
        if (s.active && s.team == 0 && s.channel + i < h.C && i >= s.skip && (local + i) - g * h.D == 0) {
            const int64_t at = s.n * h.groups + s.first / h.D + g;
            mean_out[at] = mean[i];
            rstd_out[at] = rstd;
        }
        scale[i] *= rstd;
        shift[i] = fmaf(-low, scale[i], shift[i]);
    }
    if (!s.active)
        return;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (s.team + j * h.teams >= h.L)
            break;
        unpack_again(r[j]);
        float v[GROUP];
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            v[i] = activated<ACT>(fmaf(raw_value(r[j], i) - mean[i], scale[i], shift[i]));
        store_row(h, y + s.base + j * (h.teams * h.C), v);
    }
}

// totals: dz and dz (x - mean) rstd of each sample and channel (or, of one sample,
// dbeta and dgamma themselves).
template <typename T, int ACT, int NT, int K>
__global__ __launch_bounds__(NT) void held_backward_kernel(const T* __restrict__ dy, const T* __restrict__ x, Inputs in,
                                                           Map h, T* __restrict__ dx, Pair* __restrict__ totals,
                                                           float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    extern __shared__ float lds[];
    const int64_t b = on_one_die(h.work);
    if (b < 0)
        return;
    const Spot s = spot_of(h, b);
    const int channels = h.cols * GROUP, local = s.channel - s.first;
    float* const sums = lds;                                         // of the groups
    Pair* const parts = reinterpret_cast<Pair*>(lds + 2 * h.span);   // of the channels
    Raw<T> rx[K], rd[K];
    hold(x, h, s, rx);
    hold(dy, h, s, rd);
    Lines l;
    float rstd[GROUP] = {};
    load_lines(h, s, in, l, rstd);
    float c[2][GROUP] = {};
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (s.active && s.team + j * h.teams < h.L) {
            float v[GROUP], d[GROUP], dz[GROUP];
            values_of(rx[j], v);
            values_of(rd[j], dz);
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                d[i] = v[i] - l.mean[i];
            slopes<ACT>(h, s, in, l, v, d, dz);
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                c[0][i] += dz[i];
                c[1][i] = fmaf(dz[i], d[i], c[1][i]);
            }
        }
    }
    // Each channel's sums over the workgroup's rows ...
    int row = s.team;
    bool writes = s.active;
    if (h.fold) {
        for (int m = h.cols; m < 64; m <<= 1)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < GROUP; ++i)
                    c[k][i] += __shfl_xor(c[k][i], m);
        row = threadIdx.x >> 6;
        writes = s.active && (threadIdx.x & 63) < h.cols;
    }
    if (writes) {
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            if (i >= s.skip)
                parts[row * channels + local + i] = Pair{c[0][i], c[1][i] * rstd[i]};
    }
    __syncthreads();
    const int rows = h.fold ? NT / 64 : h.teams;
    for (int k = threadIdx.x; k < channels; k += NT) {
        if (s.first + k >= h.C)
            continue;
        Pair t{0.f, 0.f};
        for (int q = 0; q < rows; ++q) {
            t.a += parts[q * channels + k].a;
            t.b += parts[q * channels + k].b;
        }
        if (h.N == 1) {
            dbeta[s.first + k] = t.a;
            dgamma[s.first + k] = t.b;
        } else {
            totals[s.n * h.C + s.first + k] = t;
        }
        parts[k] = t;     // (only this thread reads column k)
    }
    __syncthreads();
    // ... and each group's averages of g = gamma dz and of g n.
    const double count = static_cast<double>(h.L) * static_cast<double>(h.D);
    for (int g = static_cast<int>(threadIdx.x) / h.lanes; g < h.span; g += NT / h.lanes) {
        double a1 = 0.0, a2 = 0.0;
        for (int q = threadIdx.x & (h.lanes - 1); q < h.D; q += h.lanes) {
            const double w = in.gamma[s.first + g * h.D + q];
            a1 += w * parts[g * h.D + q].a;
            a2 += w * parts[g * h.D + q].b;
        }
        for (int m = 1; m < h.lanes; m <<= 1) {
            a1 += __shfl_xor(a1, m);
            a2 += __shfl_xor(a2, m);
        }
        if ((threadIdx.x & (h.lanes - 1)) == 0) {
            sums[2 * g] = static_cast<float>(a1 / count);
            sums[2 * g + 1] = static_cast<float>(a2 / count);
        }
    }
    __syncthreads();
    if (!s.active)
        return;
    // dx = rstd (gamma dz - a1 - d rstd a2)
    float k1[GROUP], k2[GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
        int g = group_of(h, local + i);
        g = g < h.span ? g : h.span - 1;
        k1[i] = -rstd[i] * sums[2 * g];
        k2[i] = -rstd[i] * rstd[i] * sums[2 * g + 1];
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (s.team + j * h.teams >= h.L)
            break;
        unpack_again(rx[j]);
        unpack_again(rd[j]);
        float v[GROUP], d[GROUP], dz[GROUP];
        values_of(rx[j], v);
        values_of(rd[j], dz);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            d[i] = v[i] - l.mean[i];
        slopes<ACT>(h, s, in, l, v, d, dz);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            v[i] = fmaf(l.scale[i], dz[i], fmaf(d[i], k2[i], k1[i]));
        store_row(h, dx + s.base + j * (h.teams * h.C), v);
    }
}

// ---------------------------------------------------------------------------
// Two to four launches, forward: mean and sum of squares about it of each chunk and
// channel; each group's mean and rstd; the result.  In two: of each chunk and group; the
// result, each workgroup with its sample's statistics from those.
// ---------------------------------------------------------------------------
constexpr int MOST_THREADS = 256;
constexpr int MOST_ROWS = 64;    // of a thread
constexpr int AT_ONCE = 4;       // rows in flight

// f(row's values) for the rows of this thread, from its `from`-th, AT_ONCE loaded
// together.
template <int M, typename T, typename F>
__device__ __forceinline__ void walk(const Map& h, const Spot& s, const T* const (&x)[M], int from, F&& f)
{
    const int64_t step = h.teams * h.C;
    int64_t at = s.base + from * step;
    for (int64_t row = s.first_row + s.team + static_cast<int64_t>(from) * h.teams; row < s.end_row;
         row += AT_ONCE * h.teams, at += AT_ONCE * step) {
        Raw<T> r[AT_ONCE][M];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            if (row + j * h.teams < s.end_row)
#pragma unroll
                for (int m = 0; m < M; ++m)
                    load_row(h, x[m] + at + j * step, r[j][m]);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            if (row + j * h.teams < s.end_row)
                f(r[j], at + j * step);
    }
}

// Sums of rows d and of the sums of squares about `from`, d a mean's distance from it:
// of any pairs, whose mean and sum of squares about it they give, in 64 bits.
struct Joined {
    double s1 = 0.0, s2 = 0.0;
    template <typename P>
    __device__ __forceinline__ void add(const P& p, double rows, double from)
    {
        const double d = p.a - from;
        s1 += rows * d;
        s2 += p.b + rows * d * d;
    }
};

// A chunk and group's mean and sum of squares about it.
struct Wide {
    double a, b;
};

// A group as the result takes it: its mean, what the mean's rounding leaves, and rstd.
// (One load.)
struct Stat {
    float mean, low, rstd;
};

__device__ __forceinline__ Stat stat_of(double mean, double var, float eps)
{
    const float m = static_cast<float>(mean);
    return Stat{m, static_cast<float>(mean - m), static_cast<float>(1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps))};   // (NaN stays)
}

// A sample's middle row.
template <typename T>
__device__ __forceinline__ const T* middle_of(const T* x, const Map& h, int64_t n)
{
    return x + (n * h.L + h.L / 2) * h.C;
}

// LATE: of each chunk and group (to `wide`), not channel (to `partial`).
//
// A mean in fp32 is its distance from a value of the group, its first channel's in the
// chunk's first row (LATE) or in the sample's middle row: rounding it costs nothing where
// the group's values lie together, far from 0.
template <typename T, bool LATE>
__global__ __launch_bounds__(MOST_THREADS) void chunk_stats_kernel(const T* __restrict__ x, Map h,
                                                                   Pair* __restrict__ partial,
                                                                   Wide* __restrict__ wide)
{
    __shared__ Pair lds[MOST_THREADS * GROUP];
    __shared__ float counts[MOST_THREADS];
    for (int64_t b = blockIdx.x; b < h.work; b += gridDim.x) {
        const Spot s = spot_of(h, b);
        const int local = s.channel - s.first, channels = h.cols * GROUP;
        const T* const near = LATE ? x + (s.n * h.L + s.first_row) * h.C : middle_of(x, h, s.n);
        float mean[GROUP] = {}, m2[GROUP] = {}, count = 0.f;
        if (s.active && s.first_row + s.team < s.end_row) {
            // differences from the thread's own first value
            Raw<T> first;
            load_row(h, x + s.base, first);
            float pivot[GROUP];
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const int c = s.channel + i < h.C ? s.channel + i : static_cast<int>(h.C) - 1;
                pivot[i] = static_cast<float>(near[group_of(h, c) * h.D]);
            }
            float s1[GROUP] = {};
            walk<1, T>(h, s, {x}, 1, [&](const Raw<T> (&r)[1], int64_t) {
#pragma unroll
                for (int i = 0; i < GROUP; ++i) {
                    const float d = raw_value(r[0], i) - raw_value(first, i);
                    s1[i] += d;
                    m2[i] = fmaf(d, d, m2[i]);
                }
            });
            count = static_cast<float>((s.end_row - s.first_row - s.team + h.teams - 1) / h.teams);
            const float inv = 1.f / count;
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const float m = s1[i] * inv, q = fmaf(-m, s1[i], m2[i]);
                mean[i] = (raw_value(first, i) - pivot[i]) + m;
                m2[i] = q < 0.f ? 0.f : q;   // (NaN stays)
            }
        }
        int row = s.team;
        bool writes = s.active;
        if (h.fold) {
            // two teams: their means' distance d moves the mean by d times the other's
            // share, and adds d^2 times the smaller count's harmonic part
            for (int m = h.cols; m < 64; m <<= 1) {
                const float other = __shfl_xor(count, m), both = count + other;
                const float share = both > 0.f ? other / both : 0.f;
#pragma unroll
                for (int i = 0; i < GROUP; ++i) {
                    const float o = __shfl_xor(mean[i], m), q = __shfl_xor(m2[i], m);
                    const float d = o - mean[i];
                    if (other > 0.f) {
                        m2[i] = count > 0.f ? fmaf(d * d, count * share, m2[i] + q) : q;
                        mean[i] = count > 0.f ? fmaf(d, share, mean[i]) : o;
                    }
                }
                count = both;
            }
            row = threadIdx.x >> 6;
            writes = s.active && (threadIdx.x & 63) < h.cols;
        }
        if (writes) {
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                if (i >= s.skip)
                    lds[row * channels + local + i] = Pair{mean[i], m2[i]};
            if (s.col == 0)
                counts[row] = count;
        }
        __syncthreads();
        // The rows of each channel, in order: the first is never empty.
        const int rows = h.fold ? (h.threads + 63) / 64 : h.teams;
        const double all = static_cast<double>(s.end_row - s.first_row);
        for (int k = threadIdx.x; k < channels; k += h.threads) {
            if (s.first + k >= h.C)
                continue;
            const double from = lds[k].a;
            Joined j;
#pragma unroll 4
            for (int w = 0; w < rows; ++w)
                if (counts[w] > 0.f)
                    j.add(lds[w * channels + k], counts[w], from);
            const double off = j.s1 / all, q = j.s2 - j.s1 * off;
            Pair* const to = LATE ? lds + k : partial + (s.n * h.chunks + s.first_row / h.rows) * h.C + s.first + k;
            *to = Pair{static_cast<float>(from + off), static_cast<float>(q < 0.0 ? 0.0 : q)};   // (NaN stays)
        }
        __syncthreads();
        if constexpr (LATE) {
            const int lane = threadIdx.x & (h.lanes - 1), D = h.D;
            for (int g = static_cast<int>(threadIdx.x) / h.lanes; g < h.groups; g += h.threads / h.lanes) {
                const Pair* const of = lds + g * D;
                const double from = of[0].a, count = all * D;
                Joined j;
                for (int c = lane; c < D; c += h.lanes)
                    j.add(of[c], all, from);
                for (int m = 1; m < h.lanes; m <<= 1) {
                    j.s1 += __shfl_xor(j.s1, m);
                    j.s2 += __shfl_xor(j.s2, m);
                }
                const double off = j.s1 / count, q = j.s2 - j.s1 * off;
                if (lane == 0)
                    wide[(s.n * h.chunks + s.first_row / h.rows) * h.groups + g] =
                        Wide{static_cast<float>(near[g * D]) + (from + off), q < 0.0 ? 0.0 : q};
            }
            __syncthreads();
        }
    }
}

// A sum over TEAM threads: a wave, or the workgroup.
template <int TEAM>
__device__ __forceinline__ double team_sum(double v, double* lds)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        v += __shfl_xor(v, d);
    if constexpr (TEAM > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int i = 0; i < TEAM / 64; ++i)
            v += lds[i];
    }
    return v;
}

// TEAM threads a group.
template <int TEAM, typename T>
__global__ __launch_bounds__(SUM_THREADS) void group_stats_kernel(const Pair* __restrict__ partial,
                                                                  const T* __restrict__ x, Map h, float eps,
                                                                  Stat* __restrict__ stats,
                                                                  float* __restrict__ mean_out,
                                                                  float* __restrict__ rstd_out)
{
    __shared__ double lds[SUM_THREADS / 64];
    constexpr int TEAMS = SUM_THREADS / TEAM;
    const int t = threadIdx.x % TEAM;
    const uint32_t D = h.D;
    const int64_t pairs = h.chunks * h.D;
    const double count = static_cast<double>(h.L) * static_cast<double>(h.D);
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * TEAMS + threadIdx.x / TEAM; q < h.N * h.groups;
         q += static_cast<int64_t>(gridDim.x) * TEAMS) {
        const int64_t n = q / h.groups;
        const Pair* at = partial + n * h.chunks * h.C + (q - n * h.groups) * h.D;
        const double from = at->a, middle = static_cast<float>(middle_of(x, h, n)[(q - n * h.groups) * h.D]);
        Joined j;
#pragma unroll 4
        for (int64_t i = t; i < pairs; i += TEAM) {
            const uint32_t chunk = static_cast<uint32_t>(i) / D, c = static_cast<uint32_t>(i) - chunk * D;
            j.add(at[chunk * h.C + c], static_cast<double>(chunk + 1 < h.chunks ? h.rows : h.L - chunk * h.rows), from);
        }
        j.s1 = team_sum<TEAM>(j.s1, lds) / count;
        j.s2 = team_sum<TEAM>(j.s2, lds) / count - j.s1 * j.s1;
        if (t == 0) {
            const Stat stat = stat_of(middle + (from + j.s1), j.s2, eps);
            stats[q] = stat;
            mean_out[q] = stat.mean;
            rstd_out[q] = stat.rstd;
        }
    }
}

// The chunks of one sample and TILE channels, TILE_SLICES threads a channel:
// f(chunk, pair) for this thread's.
constexpr int TILE = 16, TILE_SLICES = SUM_THREADS / TILE;

template <typename F>
__device__ __forceinline__ void each_chunk(const Pair* __restrict__ partial, const Map& h, int64_t n, int64_t channel,
                                           F&& f)
{
    if (channel >= h.C)
        return;
#pragma unroll 4
    for (int64_t k = threadIdx.x / TILE; k < h.chunks; k += TILE_SLICES)
        f(k, partial[(n * h.chunks + k) * h.C + channel]);
}

// The sum over a channel's threads.
__device__ __forceinline__ double slice_sum(double v, double* lds)
{
    __syncthreads();
    lds[threadIdx.x] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < TILE_SLICES; ++i)
        v += lds[threadIdx.x % TILE + i * TILE];
    return v;
}

// Each sample and channel's mean and sum of squares about it from those of its chunks:
// where a group's pairs are many.
__global__ __launch_bounds__(SUM_THREADS) void join_chunks_kernel(const Pair* __restrict__ partial, Map h,
                                                                  Pair* __restrict__ joined)
{
    __shared__ double lds[SUM_THREADS];
    const int64_t tiles = ceil_div(h.C, TILE);
    for (int64_t q = blockIdx.x; q < h.N * tiles; q += gridDim.x) {
        const int64_t n = q / tiles, channel = (q - n * tiles) * TILE + threadIdx.x % TILE;
        const double from = channel < h.C ? partial[n * h.chunks * h.C + channel].a : 0.f;
        Joined j;
        each_chunk(partial, h, n, channel, [&](int64_t k, const Pair& p) {
            j.add(p, static_cast<double>(k + 1 < h.chunks ? h.rows : h.L - k * h.rows), from);
        });
        j.s1 = slice_sum(j.s1, lds);
        j.s2 = slice_sum(j.s2, lds) - j.s1 * j.s1 / static_cast<double>(h.L);
        if (threadIdx.x < TILE && channel < h.C)
            joined[n * h.C + channel] = Pair{static_cast<float>(from + j.s1 / static_cast<double>(h.L)),
                                             static_cast<float>(j.s2 < 0.0 ? 0.0 : j.s2)};
    }
}

// What a sample's groups make of their chunks (`wide`), in each workgroup of the result:
// a thread a group and one of `slices` of the chunks; add(sums, chunk's, k, from),
// `from` being the first chunk's, and finish(group, sums, from) by one thread.
constexpr int LATE_EACH = 8, LATE_ROUNDS = 2;   // chunks of a thread in flight together, times

template <typename A, typename F>
__device__ __forceinline__ void join_late(const Wide* __restrict__ wide, const Map& h, double* lds, A&& add, F&& finish)
{
    const int groups = static_cast<int>(h.groups), chunks = static_cast<int>(h.chunks);
    const int slice = static_cast<int>(threadIdx.x) / groups, g = static_cast<int>(threadIdx.x) - slice * groups;
    double from = 0.0;
    Joined j;
    if (slice < h.slices)
        from = wide[g].a;
    for (int first = slice; slice < h.slices && first < chunks; first += LATE_EACH * h.slices) {
        Wide w[LATE_EACH];
#pragma unroll
        for (int i = 0; i < LATE_EACH; ++i)
            if (first + i * h.slices < chunks)
                w[i] = wide[(first + i * h.slices) * groups + g];
#pragma unroll
        for (int i = 0; i < LATE_EACH; ++i)
            if (first + i * h.slices < chunks)
                add(j, w[i], first + i * h.slices, from);
    }
    lds[2 * threadIdx.x] = j.s1;
    lds[2 * threadIdx.x + 1] = j.s2;
    __syncthreads();
    if (slice == 0) {
        for (int i = 1; i < h.slices; ++i) {
            j.s1 += lds[2 * (i * groups + g)];
            j.s2 += lds[2 * (i * groups + g) + 1];
        }
        finish(g, j, from);
    }
    __syncthreads();
}

// LATE: from the chunks' statistics; the workgroup of a sample's first rows writes the
// groups'.
template <typename T, int ACT, bool LATE>
__global__ __launch_bounds__(MOST_THREADS) void forward_kernel(const T* __restrict__ x,
                                                               const float* __restrict__ gamma,
                                                               const float* __restrict__ beta, Map h,
                                                               T* __restrict__ y, const Wide* __restrict__ wide,
                                                               const Stat* __restrict__ stats, float eps,
                                                               float* __restrict__ mean_out,
                                                               float* __restrict__ rstd_out)
{
    __shared__ double lds[LATE ? 2 * MOST_THREADS : 1];
    __shared__ Stat late[LATE ? MOST_THREADS : 1];
    for (int64_t b = blockIdx.x; b < h.work; b += gridDim.x) {
        const Spot s = spot_of(h, h.work - 1 - b);   // last read, first read again
        if constexpr (LATE) {
            __syncthreads();   // what the last turn left has been read
            const double D = h.D, inv = 1.0 / (static_cast<double>(h.L) * D);
            const int last = static_cast<int>(h.chunks) - 1, rows = static_cast<int>(h.rows);
            const int rest = static_cast<int>(h.L - last * h.rows);
            join_late(wide + s.n * h.chunks * h.groups, h, lds,
                      [&](Joined& j, const Wide& w, int k, double from) {
                          j.add(w, D * static_cast<double>(k < last ? rows : rest), from);
                      },
                      [&](int g, const Joined& j, double from) {
                          const double off = j.s1 * inv, var = j.s2 * inv - off * off;
                          late[g] = stat_of(from + off, var, eps);
                      });
            if (s.first_row == 0 && threadIdx.x < h.groups) {
                mean_out[s.n * h.groups + threadIdx.x] = late[threadIdx.x].mean;
                rstd_out[s.n * h.groups + threadIdx.x] = late[threadIdx.x].rstd;
            }
        }
        if (!s.active)
            continue;
        Lines l;
        load_weights(h, s, gamma, l.scale);
        load_weights(h, s, beta, l.shift);
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            const int c = s.channel + i < h.C ? s.channel + i : static_cast<int>(h.C) - 1, g = group_of(h, c);
            const Stat t = LATE ? late[g] : stats[s.n * h.groups + g];
            l.mean[i] = t.mean;
            l.scale[i] *= t.rstd;
            l.shift[i] = fmaf(-t.low, l.scale[i], l.shift[i]);
        }
        walk<1, T>(h, s, {x}, 0, [&](const Raw<T> (&r)[1], int64_t at) {
            float v[GROUP];
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] = activated<ACT>(fmaf(raw_value(r[0], i) - l.mean[i], l.scale[i], l.shift[i]));
            stream_row(h, y + at, v);
        });
    }
}

// ---------------------------------------------------------------------------
// Two to four launches, backward: sums of dz and dz n of each chunk and channel; of each
// sample and channel, and each group's averages; the result, and dgamma and dbeta.  In
// two, the chunks' groups are summed up where the chunks are, as in the forward pass.
// ---------------------------------------------------------------------------
// LATE: of each chunk and group too, weighted by gamma (to `wide`).
template <typename T, int ACT, bool LATE>
__global__ __launch_bounds__(MOST_THREADS) void chunk_sums_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                                  Inputs in, Map h, Pair* __restrict__ partial,
                                                                  Wide* __restrict__ wide)
{
    __shared__ Pair lds[MOST_THREADS * GROUP];
    for (int64_t b = blockIdx.x; b < h.work; b += gridDim.x) {
        const Spot s = spot_of(h, b);
        const int local = s.channel - s.first, channels = h.cols * GROUP;
        float c[2][GROUP] = {}, rstd[GROUP] = {};
        if (s.active) {
            Lines l;
            load_lines(h, s, in, l, rstd);
            walk<2, T>(h, s, {x, dy}, 0, [&](const Raw<T> (&r)[2], int64_t) {
                float v[GROUP], d[GROUP], dz[GROUP];
                values_of(r[0], v);
                values_of(r[1], dz);
#pragma unroll
                for (int i = 0; i < GROUP; ++i)
                    d[i] = v[i] - l.mean[i];
                slopes<ACT>(h, s, in, l, v, d, dz);
#pragma unroll
                for (int i = 0; i < GROUP; ++i) {
                    c[0][i] += dz[i];
                    c[1][i] = fmaf(dz[i], d[i], c[1][i]);
                }
            });
        }
        int row = s.team;
        bool writes = s.active;
        if (h.fold) {
            for (int m = h.cols; m < 64; m <<= 1)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < GROUP; ++i)
                        c[k][i] += __shfl_xor(c[k][i], m);
            row = threadIdx.x >> 6;
            writes = s.active && (threadIdx.x & 63) < h.cols;
        }
        if (writes) {
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                if (i >= s.skip)
                    lds[row * channels + local + i] = Pair{c[0][i], c[1][i] * rstd[i]};
        }
        __syncthreads();
        const int rows = h.fold ? (h.threads + 63) / 64 : h.teams;
        for (int k = threadIdx.x; k < channels; k += h.threads) {
            if (s.first + k >= h.C)
                continue;
            Pair t{0.f, 0.f};
            for (int w = 0; w < rows; ++w) {
                t.a += lds[w * channels + k].a;
                t.b += lds[w * channels + k].b;
            }
            partial[(s.n * h.chunks + s.first_row / h.rows) * h.C + s.first + k] = t;
            if (LATE)
                lds[k] = t;
        }
        __syncthreads();
        if constexpr (LATE) {
            const int lane = threadIdx.x & (h.lanes - 1), D = h.D;
            for (int g = static_cast<int>(threadIdx.x) / h.lanes; g < h.groups; g += h.threads / h.lanes) {
                double s1 = 0.0, s2 = 0.0;
                for (int c = g * D + lane; c < g * D + D; c += h.lanes) {
                    const double w = in.gamma[c];
                    s1 += w * lds[c].a;
                    s2 += w * lds[c].b;
                }
                for (int m = 1; m < h.lanes; m <<= 1) {
                    s1 += __shfl_xor(s1, m);
                    s2 += __shfl_xor(s2, m);
                }
                if (lane == 0)
                    wide[(s.n * h.chunks + s.first_row / h.rows) * h.groups + g] = Wide{s1, s2};
            }
            __syncthreads();
        }
    }
}

// Narrow groups (up to NARROW channels), one workgroup a group of one sample: its
// channels' sums over the chunks, a channel a lane of `lanes`, and its averages.
constexpr int NARROW = 64;

__global__ __launch_bounds__(SUM_THREADS) void join_sums_kernel(const Pair* __restrict__ partial, Map h,
                                                                const float* __restrict__ gamma,
                                                                Pair* __restrict__ totals, Pair* __restrict__ averages)
{
    __shared__ double lds[SUM_THREADS * 2];
    int lanes = 1;
    while (lanes < h.D)
        lanes *= 2;
    const int slices = SUM_THREADS / lanes, lane = threadIdx.x & (lanes - 1), slice = threadIdx.x / lanes;
    const double count = static_cast<double>(h.L) * static_cast<double>(h.D);
    for (int64_t q = blockIdx.x; q < h.N * h.groups; q += gridDim.x) {
        const int64_t n = q / h.groups, channel = (q - n * h.groups) * h.D + lane;
        double s1 = 0.0, s2 = 0.0;
        if (lane < h.D)
#pragma unroll 4
            for (int64_t k = slice; k < h.chunks; k += slices) {
                const Pair p = partial[(n * h.chunks + k) * h.C + channel];
                s1 += p.a;
                s2 += p.b;
            }
        __syncthreads();
        lds[threadIdx.x * 2] = s1;
        lds[threadIdx.x * 2 + 1] = s2;
        __syncthreads();
        if (slice != 0)
            continue;   // (the rest within one wave)
        for (int k = 1; k < slices; ++k) {
            s1 += lds[(k * lanes + lane) * 2];
            s2 += lds[(k * lanes + lane) * 2 + 1];
        }
        double a1 = 0.0, a2 = 0.0;
        if (lane < h.D) {
            totals[n * h.C + channel] = Pair{static_cast<float>(s1), static_cast<float>(s2)};
            a1 = gamma[channel] * s1;
            a2 = gamma[channel] * s2;
        }
        for (int m = 1; m < lanes; m <<= 1) {
            a1 += __shfl_xor(a1, m);
            a2 += __shfl_xor(a2, m);
        }
        if (lane == 0)
            averages[q] = Pair{static_cast<float>(a1 / count), static_cast<float>(a2 / count)};
    }
}

// Wide ones: the sums of each sample and channel, then a workgroup a group.
__global__ __launch_bounds__(SUM_THREADS) void join_channels_kernel(const Pair* __restrict__ partial, Map h,
                                                                    Pair* __restrict__ totals)
{
    __shared__ double lds[SUM_THREADS];
    const int64_t tiles = ceil_div(h.C, TILE);
    for (int64_t q = blockIdx.x; q < h.N * tiles; q += gridDim.x) {
        const int64_t n = q / tiles, channel = (q - n * tiles) * TILE + threadIdx.x % TILE;
        double s1 = 0.0, s2 = 0.0;
        each_chunk(partial, h, n, channel, [&](int64_t, const Pair& p) {
            s1 += p.a;
            s2 += p.b;
        });
        s1 = slice_sum(s1, lds);
        s2 = slice_sum(s2, lds);
        if (threadIdx.x < TILE && channel < h.C)
            totals[n * h.C + channel] = Pair{static_cast<float>(s1), static_cast<float>(s2)};
    }
}

__global__ __launch_bounds__(SUM_THREADS) void average_kernel(const Pair* __restrict__ totals, Map h,
                                                              const float* __restrict__ gamma,
                                                              Pair* __restrict__ averages)
{
    __shared__ double lds[SUM_THREADS / 64];
    const double count = static_cast<double>(h.L) * static_cast<double>(h.D);
    for (int64_t q = blockIdx.x; q < h.N * h.groups; q += gridDim.x) {
        const int64_t n = q / h.groups, first = (q - n * h.groups) * h.D;
        double a1 = 0.0, a2 = 0.0;
#pragma unroll 4
        for (int64_t c = threadIdx.x; c < h.D; c += SUM_THREADS) {
            const Pair p = totals[n * h.C + first + c];
            const double w = gamma[first + c];
            a1 += w * p.a;
            a2 += w * p.b;
        }
        a1 = team_sum<SUM_THREADS>(a1, lds);
        a2 = team_sum<SUM_THREADS>(a2, lds);
        if (threadIdx.x == 0)
            averages[q] = Pair{static_cast<float>(a1 / count), static_cast<float>(a2 / count)};
    }
}

// dgamma and dbeta from the samples' totals, SUM_COLS channels a workgroup of
// `threads` (64 at least; lds: a pair for each).
constexpr int SUM_COLS = 16;

__device__ __forceinline__ void sum_samples(const Pair* __restrict__ totals, int64_t N, int64_t C, int64_t first,
                                            int threads, double* lds, float* __restrict__ dgamma,
                                            float* __restrict__ dbeta)
{
    const int slices = threads / SUM_COLS;
    const int lane = threadIdx.x % SUM_COLS, w = threadIdx.x / SUM_COLS;
    const int64_t channel = first + lane;
    double s1 = 0.0, s2 = 0.0;
    if (channel < C)
#pragma unroll 4
        for (int64_t i = w; i < N; i += slices) {
            const Pair p = totals[i * C + channel];
            s1 += p.a;
            s2 += p.b;
        }
    lds[threadIdx.x * 2] = s1;
    lds[threadIdx.x * 2 + 1] = s2;
    __syncthreads();
    if (w == 0 && channel < C) {
        for (int i = 1; i < slices; ++i) {
            s1 += lds[(i * SUM_COLS + lane) * 2];
            s2 += lds[(i * SUM_COLS + lane) * 2 + 1];
        }
        dbeta[channel] = static_cast<float>(s1);
        dgamma[channel] = static_cast<float>(s2);
    }
}

__global__ __launch_bounds__(SUM_THREADS) void weights_kernel(const Pair* __restrict__ totals, int64_t N, int64_t C,
                                                              float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ double lds[SUM_THREADS * 2];
    sum_samples(totals, N, C, static_cast<int64_t>(blockIdx.x) * SUM_COLS, SUM_THREADS, lds, dgamma, dbeta);
}

// totals: of each sample and channel, or (LATE) chunk and channel.
template <typename T, int ACT, bool LATE>
__global__ __launch_bounds__(MOST_THREADS) void backward_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                                Inputs in, Map h, const Pair* __restrict__ averages,
                                                                T* __restrict__ dx, const Pair* __restrict__ totals,
                                                                float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                                unsigned sums, const Wide* __restrict__ wide)
{
    __shared__ double lds[MOST_THREADS * 2];
    __shared__ Pair late[LATE ? MOST_THREADS : 1];
    if (blockIdx.x < sums) {   // the first workgroups, not the last: theirs is a chain of loads
        sum_samples(totals, LATE ? h.N * h.chunks : h.N, h.C, static_cast<int64_t>(blockIdx.x) * SUM_COLS, h.threads,
                    lds, dgamma, dbeta);
        return;
    }
    for (int64_t b = blockIdx.x - sums; b < h.work; b += gridDim.x - sums) {
        const Spot s = spot_of(h, h.work - 1 - b);   // last read, first read again
        if constexpr (LATE) {
            const double inv = 1.0 / (static_cast<double>(h.L) * static_cast<double>(h.D));
            __syncthreads();   // what the last turn left has been read
            join_late(wide + s.n * h.chunks * h.groups, h, lds,
                      [](Joined& j, const Wide& w, int, double) {
                          j.s1 += w.a;
                          j.s2 += w.b;
                      },
                      [&](int g, const Joined& j, double) {
                          late[g] = Pair{static_cast<float>(j.s1 * inv), static_cast<float>(j.s2 * inv)};
                      });
        }
        if (!s.active)
            continue;
        Lines l;
        float rstd[GROUP], k1[GROUP], k2[GROUP];
        load_lines(h, s, in, l, rstd);
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            const int c = s.channel + i < h.C ? s.channel + i : static_cast<int>(h.C) - 1;
            const Pair a = LATE ? late[group_of(h, c)] : averages[s.n * h.groups + group_of(h, c)];
            k1[i] = -rstd[i] * a.a;
            k2[i] = -rstd[i] * rstd[i] * a.b;
        }
        walk<2, T>(h, s, {x, dy}, 0, [&](const Raw<T> (&r)[2], int64_t at) {
            float v[GROUP], d[GROUP], dz[GROUP];
            values_of(r[0], v);
            values_of(r[1], dz);
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                d[i] = v[i] - l.mean[i];
            slopes<ACT>(h, s, in, l, v, d, dz);
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] = fmaf(l.scale[i], dz[i], fmaf(d[i], k2[i], k1[i]));
            stream_row(h, dx + at, v);
        });
    }
}

// ---------------------------------------------------------------------------
// Launches.
// ---------------------------------------------------------------------------
int32_t gcd(int64_t a, int64_t b) { return static_cast<int32_t>(b ? gcd(b, a % b) : a); }

Map map_of(int64_t N, int64_t L, int64_t C, int64_t groups, int64_t cols, int64_t threads)
{
    Map h{};
    h.N = N;
    h.L = L;
    h.C = C;
    h.groups = groups;
    h.D = static_cast<int32_t>(C / groups);
    h.inv_D = 1.f / static_cast<float>(h.D);
    h.cols = static_cast<int32_t>(cols);
    h.sides = static_cast<int32_t>(ceil_div(ceil_div(C, GROUP), cols));
    h.teams = static_cast<int32_t>(threads / cols);
    h.threads = static_cast<int32_t>(threads);
    h.piece = gcd(h.D, GROUP);
    h.shift = h.piece == 8 ? 3 : h.piece >> 1;   // 1, 2, 4
    h.fold = cols <= 64 && (cols & (cols - 1)) == 0;
    h.rows = L;
    h.chunks = 1;
    h.work = N * h.sides;
    return h;
}

// The cut of the three launches: eight workgroups a CU, where each thread then has
// at least four rows and at most MOST_ROWS.  (Chunks of 64 rows at least, while that
// leaves every CU one: forward 1 x 12544 x 2048 bf16 57 -> 47 us, but backward 4 x 9000
// x 1000 fp32 143 -> 156 and 17 x 1225 x 288 fp32 30 -> 33.)
Map cut(int64_t N, int64_t L, int64_t C, int64_t groups)
{
    const int64_t all = ceil_div(C, GROUP), sides = ceil_div(all, MOST_THREADS), cols = ceil_div(all, sides);
    int64_t teams = std::max<int64_t>(1, std::min<int64_t>(MOST_THREADS / cols, L));
    if (cols <= 64 && (cols & (cols - 1)) == 0)   // whole waves, which are joined by shuffles
        teams = ceil_div(teams * cols, 64) * 64 / cols;
    Map h = map_of(N, L, C, groups, cols, ceil_div(cols * teams, 64) * 64);
    h.teams = static_cast<int32_t>(teams);
    const int64_t wanted = std::max<int64_t>(1, ceil_div(8 * 256, std::max<int64_t>(1, N * h.sides)));
    const int64_t each = std::min<int64_t>(MOST_ROWS, std::max<int64_t>(4, ceil_div(L, wanted * teams)));
    h.rows = std::min<int64_t>(L, each * teams);
    h.chunks = ceil_div(L, h.rows);
    h.work = N * h.chunks * h.sides;
    h.lanes = 1;
    while (h.lanes < 64 && 2 * h.lanes * groups <= h.threads)
        h.lanes *= 2;
    h.slices = static_cast<int32_t>(std::max<int64_t>(1, h.threads / groups));
    return h;
}

// Whether each workgroup of the result joins its sample's groups itself (join_late),
// which leaves out a launch: where a row is one workgroup's and a group's chunks are few
// to a thread.  Forward, three launches and two: 2 x 1225 x 288 fp32 in 32 groups 14.9
// and 12.1 us, 17 x 1225 x 288 26.0 and 22.9, 4 x 9000 x 1000 fp32 in 8 98 and 89, 32 x
// 50176 x 64 bf16 in 32 116 and 114; with 16 chunks a thread but in one round (more
// registers) 128, with 131 chunks of 32 groups in three rounds (8 x 3136 x 320 fp32)
// 31.7 and 32.0, with one group of 2048 chunks 16.7 and 25.9.  The backward pass has
// more to do at both ends and takes it where the chip holds all workgroups at once: 60 x
// 784 x 100 bf16 in 20 21.9 and 19.4, 2 x 1225 x 288 fp32 14.4 and 12.6, but 32 x 3136 x
// 256 bf16 on 1792 workgroups 56 and 58.
constexpr int64_t LATE_FEWEST = 8, LATE_WORK = 1024;   // groups; workgroups of a backward pass
bool joins_late(int op, const Map& h)
{
    return h.sides == 1 && h.groups >= LATE_FEWEST && h.groups <= h.threads &&
           h.chunks <= LATE_ROUNDS * LATE_EACH * h.slices &&
           (op == POSEIDON_GROUP_NORM_FORWARD || h.work <= LATE_WORK);
}

// Whether the forward pass joins each channel's chunks before its groups' channels:
// where a workgroup's threads would walk more than MANY of a group's pairs.
constexpr int64_t MANY = 16;
bool joins_chunks(const Map& h) { return h.chunks > 1 && h.chunks * h.D > SUM_THREADS * MANY; }

// Threads and held rows of a workgroup.
template <int NT_, int K_>
struct Shape {
    static constexpr int NT = NT_, K = K_;
};

constexpr int SHAPES = 6;
constexpr int SHAPE_NT[SHAPES] = {256, 256, 256, 512, 512, 512};
constexpr int SHAPE_K[SHAPES] = {2, 4, 8, 8, 16, 32};

// Held values (`maps`: x, or x and dy) take at most half of a CU's registers, and 128
// of a thread's.
constexpr int64_t MOST_HELD = 512 * 128 * 4;
constexpr bool shape_fits(int K, int value_bytes, int maps) { return K * maps * value_bytes * GROUP / 4 <= 128; }

template <typename F>
hipError_t with_shape(int shape, F&& f)
{
    switch (shape) {
    case 0: return f(Shape<SHAPE_NT[0], SHAPE_K[0]>());
    case 1: return f(Shape<SHAPE_NT[1], SHAPE_K[1]>());
    case 2: return f(Shape<SHAPE_NT[2], SHAPE_K[2]>());
    case 3: return f(Shape<SHAPE_NT[3], SHAPE_K[3]>());
    case 4: return f(Shape<SHAPE_NT[4], SHAPE_K[4]>());
    default: return f(Shape<SHAPE_NT[5], SHAPE_K[5]>());
    }
}

struct Choice {
    int shape = -1;   // -1: three launches
    Map h{};
    int64_t lds = 0;
};

constexpr int64_t MOST_LDS = 65536;

// The workgroup of `shape` with `cols` columns, where a sample's groups fit it.
Choice held_as(int op, int64_t N, int64_t L, int64_t C, int64_t groups, int shape, int64_t cols)
{
    Choice q;
    const int NT = SHAPE_NT[shape];
    if (cols > NT || ceil_div(L, NT / cols) > SHAPE_K[shape])
        return q;
    Map& h = q.h;
    h = map_of(N, L, C, groups, cols, NT);
    h.span = static_cast<int32_t>(h.sides == 1 ? groups : cols * GROUP / h.D);
    h.lanes = 1;
    while (h.lanes < 64 && 2 * h.lanes * h.span <= NT)
        h.lanes *= 2;
    const int64_t rows = h.fold ? NT / 64 : h.teams;
    q.lds = 8 * (h.span + rows * h.cols * GROUP / (op == POSEIDON_GROUP_NORM_FORWARD ? h.piece : 1));
    if (q.lds <= MOST_LDS && h.work <= (int64_t(1) << 22) - XCDS)
        q.shape = shape;
    return q;
}

// Of the workgroups of whole groups that hold their share of a sample: the widest
// (rows of up to 512 bytes, or longer ones where threads would have none) that still
// give every CU one, else the narrowest; of the shapes for it, the first that fits
// (8192 x 1 x 4096 bf16 forward, an eighth of a workgroup's threads at work in rows of
// 512 bytes 742 us, all of them in rows of 4 KB 117).  What is left to the other
// launches, us held and in three of them: rows below 64 bytes, which share memory lines
// with other workgroups, in more than one round of workgroups (backward, bf16, 32 x 3136
// x 256 in rows of 16 bytes 93, 60); workgroups that fill a CU's registers, which load and store in turn, but
// for one round of them over half of the chip or more (forward, 4 x 12544 x 128 on 64
// CUs 36, 21, 32 x 3136 x 256 on 256 30, 38; backward, 2 x 1024 x 320 on 16 CUs 20,
// 15, 16 x 3136 x 256 on 256 28, 37); those that fill half of them on fewer than 64
// CUs (forward, 40 x 900 x 57 on 40 CUs 21, 16).
Choice choose(int op, int64_t N, int64_t L, int64_t C, int64_t groups, int32_t dtype)
{
    const int64_t all = ceil_div(C, GROUP), D = C / groups, bytes = dtype == POSEIDON_BF16 ? 2 : 4;
    const int64_t unit = C % GROUP ? all : D / gcd(D, GROUP);   // columns of whole groups
    const int maps = op == POSEIDON_GROUP_NORM_FORWARD ? 1 : 2;
    Choice best;
    for (int64_t cols = unit; cols <= all && cols <= 512; cols += unit) {
        if (all % cols)
            continue;
        const int64_t work = N * (all / cols), wide = cols * GROUP * bytes;
        if (best.shape >= 0 && (work < 256 || (wide > 512 && best.h.teams <= L)))
            break;
        if (wide < 64 && cols < all && work > 256)
            continue;
        for (int shape = 0; shape < SHAPES; ++shape) {
            const int64_t held = SHAPE_NT[shape] * SHAPE_K[shape] * GROUP * bytes * maps;   // bytes
            if (held > MOST_HELD || (held > MOST_HELD / 2 && (work < 128 || work > 256)) ||
                (held > MOST_HELD / 4 && work < 64))
                continue;
            const Choice q = held_as(op, N, L, C, groups, shape, cols);
            if (q.shape >= 0) {
                best = q;
                break;
            }
        }
    }
    return best;
}

unsigned held_grid(const Map& h) { return static_cast<unsigned>(ceil_div(h.work, XCDS) * XCDS); }

// Within a launch's limit of 2^32 threads: the kernels walk what is over.
unsigned grid_for(int64_t work) { return static_cast<unsigned>(std::min<int64_t>(work, 1 << 20)); }

template <typename T>
constexpr int32_t type_of()
{
    return sizeof(T) == 2 ? POSEIDON_BF16 : POSEIDON_F32;
}

template <typename F>
void with_act(int32_t act, F&& f)
{
    switch (act) {
    case POSEIDON_ACT_RELU: f(std::integral_constant<int, POSEIDON_ACT_RELU>()); break;
    case POSEIDON_ACT_SILU: f(std::integral_constant<int, POSEIDON_ACT_SILU>()); break;
    default: f(std::integral_constant<int, POSEIDON_ACT_NONE>());
    }
}

template <typename T>
hipError_t forward_typed(int64_t N, int64_t L, int64_t C, int64_t groups, const T* x, const float* gamma,
                         const float* beta, float eps, int32_t act, T* y, float* mean, float* rstd, void* ws,
                         hipStream_t s)
{
    const Choice q = choose(POSEIDON_GROUP_NORM_FORWARD, N, L, C, groups, type_of<T>());
    if (q.shape >= 0)
        return with_shape(q.shape, [&](auto shape) {
            with_act(act, [&](auto a) {
                constexpr int NT = decltype(shape)::NT, K = decltype(shape)::K;
                if constexpr (shape_fits(K, sizeof(T), 1))
                    held_forward_kernel<T, decltype(a)::value, NT, K><<<held_grid(q.h), NT, q.lds, s>>>(
                        x, gamma, beta, q.h, eps, y, mean, rstd);
            });
            return hipGetLastError();
        });
    const Map h = cut(N, L, C, groups);
    auto result = [&](auto late, const Wide* wide, const Stat* stats) {
        with_act(act, [&](auto a) {
            forward_kernel<T, decltype(a)::value, decltype(late)::value><<<grid_for(h.work), h.threads, 0, s>>>(
                x, gamma, beta, h, y, wide, stats, eps, mean, rstd);
        });
        return hipGetLastError();
    };
    if (joins_late(POSEIDON_GROUP_NORM_FORWARD, h)) {
        Wide* const wide = static_cast<Wide*>(ws);
        chunk_stats_kernel<T, true><<<grid_for(h.work), h.threads, 0, s>>>(x, h, nullptr, wide);
        const hipError_t rc = hipGetLastError();
        return rc != hipSuccess ? rc : result(std::true_type(), wide, nullptr);
    }
    Pair* const partial = static_cast<Pair*>(ws);
    Stat* const stats_of = reinterpret_cast<Stat*>(partial + N * h.chunks * C + (joins_chunks(h) ? N * C : 0));
    chunk_stats_kernel<T, false><<<grid_for(h.work), h.threads, 0, s>>>(x, h, partial, nullptr);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess)
        return rc;
    const Pair* pairs_of = partial;
    Map of = h;
    if (joins_chunks(h)) {
        Pair* const joined = partial + N * h.chunks * C;
        join_chunks_kernel<<<grid_for(N * ceil_div(C, TILE)), SUM_THREADS, 0, s>>>(partial, h, joined);
        rc = hipGetLastError();
        if (rc != hipSuccess)
            return rc;
        pairs_of = joined;
        of.chunks = 1;
        of.rows = L;
    }
    const int64_t pairs = of.chunks * of.D, all = N * groups;
    auto stats = [&](auto* kernel, int team) {
        kernel<<<grid_for(ceil_div(all, SUM_THREADS / team)), SUM_THREADS, 0, s>>>(pairs_of, x, of, eps, stats_of, mean,
                                                                                   rstd);
    };
    if (pairs <= 64 * 8)
        stats(group_stats_kernel<64, T>, 64);
    else
        stats(group_stats_kernel<SUM_THREADS, T>, SUM_THREADS);
    rc = hipGetLastError();
    if (rc != hipSuccess)
        return rc;
    return result(std::false_type(), nullptr, stats_of);
}

template <typename T>
hipError_t backward_typed(int64_t N, int64_t L, int64_t C, int64_t groups, const T* dy, const T* x, const Inputs& in,
                          int32_t act, T* dx, float* dgamma, float* dbeta, void* ws, hipStream_t s)
{
    Pair* const totals = static_cast<Pair*>(ws);
    const Choice q = choose(POSEIDON_GROUP_NORM_BACKWARD, N, L, C, groups, type_of<T>());
    hipError_t rc = hipSuccess;
    if (N > 0 && q.shape >= 0) {
        rc = with_shape(q.shape, [&](auto shape) {
            with_act(act, [&](auto a) {
                constexpr int NT = decltype(shape)::NT, K = decltype(shape)::K;
                if constexpr (shape_fits(K, sizeof(T), 2))
                    held_backward_kernel<T, decltype(a)::value, NT, K><<<held_grid(q.h), NT, q.lds, s>>>(
                        dy, x, in, q.h, dx, totals, dgamma, dbeta);
            });
            return hipGetLastError();
        });
        if (rc != hipSuccess || N == 1)
            return rc;
    } else if (N > 0) {
        const Map h = cut(N, L, C, groups);
        const unsigned sums = static_cast<unsigned>(ceil_div(C, SUM_COLS));
        auto sums_of = [&](auto late, Pair* partial, Wide* wide) {
            with_act(act, [&](auto a) {
                chunk_sums_kernel<T, decltype(a)::value, decltype(late)::value><<<grid_for(h.work), h.threads, 0, s>>>(
                    dy, x, in, h, partial, wide);
            });
            return hipGetLastError();
        };
        auto result = [&](auto late, const Pair* of, const Pair* averages, const Wide* wide) {
            with_act(act, [&](auto a) {
                backward_kernel<T, decltype(a)::value, decltype(late)::value>
                    <<<sums + grid_for(h.work), h.threads, 0, s>>>(dy, x, in, h, averages, dx, of, dgamma, dbeta, sums,
                                                                   wide);
            });
            return hipGetLastError();
        };
        if (joins_late(POSEIDON_GROUP_NORM_BACKWARD, h)) {
            Wide* const wide = static_cast<Wide*>(ws);
            Pair* const partial = reinterpret_cast<Pair*>(wide + N * h.chunks * groups);
            rc = sums_of(std::true_type(), partial, wide);
            return rc != hipSuccess ? rc : result(std::true_type(), partial, nullptr, wide);
        }
        Pair* const averages = totals + N * C;
        Pair* const partial = averages + N * groups;
        rc = sums_of(std::false_type(), partial, nullptr);
        if (rc != hipSuccess)
            return rc;
        if (h.D <= NARROW) {
            join_sums_kernel<<<grid_for(N * groups), SUM_THREADS, 0, s>>>(partial, h, in.gamma, totals, averages);
        } else {
            join_channels_kernel<<<grid_for(N * ceil_div(C, TILE)), SUM_THREADS, 0, s>>>(partial, h, totals);
            rc = hipGetLastError();
            if (rc != hipSuccess)
                return rc;
            average_kernel<<<grid_for(N * groups), SUM_THREADS, 0, s>>>(totals, h, in.gamma, averages);
        }
        rc = hipGetLastError();
        if (rc != hipSuccess)
            return rc;
        return result(std::false_type(), totals, averages, nullptr);
    }
    weights_kernel<<<static_cast<unsigned>(ceil_div(C, SUM_COLS)), SUM_THREADS, 0, s>>>(totals, N, C, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace

int64_t group_norm_workspace(int32_t op, int64_t N, int64_t L, int64_t C, int64_t groups, int32_t dtype)
{
    const bool backward = op == POSEIDON_GROUP_NORM_BACKWARD;
    const int64_t totals = backward && N > 1 ? N * C : 0;
    if (choose(op, N, L, C, groups, dtype).shape >= 0)
        return totals * static_cast<int64_t>(sizeof(Pair));
    const Map h = cut(N, L, C, groups);
    if (joins_late(op, h))
        return N * h.chunks * (groups * static_cast<int64_t>(sizeof(Wide)) +
                               (backward ? C : 0) * static_cast<int64_t>(sizeof(Pair)));
    const int64_t pairs = N * h.chunks * C + (backward ? N * C + N * groups : joins_chunks(h) ? N * C : 0);
    return pairs * static_cast<int64_t>(sizeof(Pair)) + (backward ? 0 : N * groups * static_cast<int64_t>(sizeof(Stat)));
}

hipError_t launch_group_norm_forward(const void* x, const float* gamma, const float* beta, int64_t N, int64_t L,
                                     int64_t C, int64_t groups, int32_t dtype, float eps, int32_t act, void* y,
                                     float* mean, float* rstd, void* ws, hipStream_t stream)
{
    if (dtype == POSEIDON_BF16)
        return forward_typed(N, L, C, groups, static_cast<const __bf16*>(x), gamma, beta, eps, act,
                             static_cast<__bf16*>(y), mean, rstd, ws, stream);
    return forward_typed(N, L, C, groups, static_cast<const float*>(x), gamma, beta, eps, act, static_cast<float*>(y),
                         mean, rstd, ws, stream);
}

hipError_t launch_group_norm_backward(const void* dy, const void* x, const float* gamma, const float* beta,
                                      const float* mean, const float* rstd, int64_t N, int64_t L, int64_t C,
                                      int64_t groups, int32_t dtype, int32_t act, void* dx, float* dgamma,
                                      float* dbeta, void* ws, hipStream_t stream)
{
    const Inputs in{gamma, beta, mean, rstd};
    if (dtype == POSEIDON_BF16)
        return backward_typed(N, L, C, groups, static_cast<const __bf16*>(dy), static_cast<const __bf16*>(x), in, act,
                              static_cast<__bf16*>(dx), dgamma, dbeta, ws, stream);
    return backward_typed(N, L, C, groups, static_cast<const float*>(dy), static_cast<const float*>(x), in, act,
                          static_cast<float*>(dx), dgamma, dbeta, ws, stream);
}

}  // namespace poseidon
