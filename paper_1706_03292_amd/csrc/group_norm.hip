// Group norm with an activation, channels last, and its backward pass
// (include/poseidon.h gives the formulas).  A few operations per value, bound by
// memory: x (and dy) read, y (dx) written once each is what it cannot do without.
//
// A sample is L rows of C channels.  A workgroup takes a chunk of a sample's rows
// and up to 256 groups of eight neighbouring channels; a thread keeps its eight
// channels and walks the rows.  Three launches: sums of each chunk and channel,
// each group's statistics from them (and the weights' gradients), the result.
//
// Sums over a thread's rows (at most 64) are fp32, of differences from the first
// of its values, so that a mean far from 0 costs no accuracy; what joins threads,
// chunks and channels are means and sums of squares about them, in 64 bits.
// Nothing depends on timing.
#include "elements.h"

namespace poseidon {
namespace {

constexpr int COLS = 256;        // groups of eight channels that a workgroup holds
constexpr int MOST_THREADS = 256;
constexpr int MOST_ROWS = 64;    // of a thread
constexpr int SUM_THREADS = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How the rows and channels are cut: columns of eight channels, teams of threads
// that hold one row each, rows a chunk.
struct Cut {
    int64_t N, L, C, groups, D;   // D channels a group
    int64_t rows;                 // of a chunk
    int32_t chunks, cols, sides;  // chunks of a sample; columns and workgroups across
    int32_t teams, threads;
};

Cut make_cut(int64_t N, int64_t L, int64_t C, int64_t groups)
{
    Cut c{N, L, C, groups, C / groups, 0, 0, 0, 0, 0, 0};
    const int64_t all = ceil_div(C, GROUP);
    c.sides = static_cast<int32_t>(ceil_div(all, COLS));
    c.cols = static_cast<int32_t>(ceil_div(all, c.sides));
    c.teams = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(MOST_THREADS / c.cols, L)));
    c.threads = static_cast<int32_t>(ceil_div(static_cast<int64_t>(c.cols) * c.teams, 64) * 64);
    // Eight workgroups a CU, where each thread then has at least four rows.
    const int64_t wanted = std::max<int64_t>(1, ceil_div(8 * 256, std::max<int64_t>(1, N * c.sides)));
    const int64_t per_thread = std::min<int64_t>(MOST_ROWS, std::max<int64_t>(4, ceil_div(L, wanted * c.teams)));
    c.rows = std::min<int64_t>(L, per_thread * c.teams);
    c.chunks = static_cast<int32_t>(ceil_div(L, std::max<int64_t>(1, c.rows)));
    return c;
}

// The place of a workgroup: sample, chunk and side, walked in one dimension.
struct Place {
    int64_t n, chunk, first_row, end_row;
    int64_t channel;     // of this thread; past the last: at least C
    int team;
    bool active;
};

__device__ __forceinline__ Place place_of(const Cut& c, int64_t b)
{
    Place p;
    const int64_t side = b % c.sides;
    b /= c.sides;
    p.chunk = b % c.chunks;
    p.n = b / c.chunks;
    p.first_row = p.chunk * c.rows;
    p.end_row = p.first_row + c.rows < c.L ? p.first_row + c.rows : c.L;
    const int t = threadIdx.x;
    p.team = t / c.cols;
    p.channel = (side * c.cols + t % c.cols) * GROUP;
    p.active = p.team < c.teams && p.channel < c.C;
    return p;
}

// A pair of sums for each chunk and channel.
struct Pair {
    float a, b;
};

__device__ __forceinline__ Pair* pair_at(Pair* partial, const Cut& c, int64_t n, int64_t chunk, int64_t channel)
{
    return partial + (n * c.chunks + chunk) * c.C + channel;
}

// The eight values of a group's array at this thread's channels.
__device__ __forceinline__ void per_channel(const float* of_groups, const Cut& c, int64_t n, int64_t channel,
                                            float (&v)[GROUP])
{
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
        v[i] = channel + i < c.C ? of_groups[n * c.groups + (channel + i) / c.D] : 0.f;
}

// ---------------------------------------------------------------------------
// Forward: mean and sum of squares about it of each chunk and channel.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(MOST_THREADS) void chunk_stats_kernel(const T* __restrict__ x, Cut c, int64_t work,
                                                                   Pair* __restrict__ partial)
{
    __shared__ Pair lds[MOST_THREADS * GROUP];
    for (int64_t b = blockIdx.x; b < work; b += gridDim.x) {
        const Place p = place_of(c, b);
        const int64_t left = c.C - p.channel;
        const int64_t first = p.first_row + p.team;
        if (p.active && first < p.end_row) {
            const T* at = x + (p.n * c.L + first) * c.C + p.channel;
            float pivot[GROUP], s1[GROUP] = {}, s2[GROUP] = {}, v[GROUP];
            load_some(at, left, pivot);
            for (int64_t r = first + c.teams; r < p.end_row; r += c.teams) {
                at += c.teams * c.C;
                load_some(at, left, v);
#pragma unroll
                for (int i = 0; i < GROUP; ++i) {
                    const float d = v[i] - pivot[i];
                    s1[i] += d;
                    s2[i] = fmaf(d, d, s2[i]);
                }
            }
            const float inv = 1.f / static_cast<float>((p.end_row - first + c.teams - 1) / c.teams);
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const float m = s1[i] * inv;
                lds[threadIdx.x * GROUP + i] = Pair{pivot[i] + m, fmaxf(fmaf(-m, s1[i], s2[i]), 0.f)};
            }
        }
        __syncthreads();
        // The teams of each channel, in order.
        const int64_t rows = p.end_row - p.first_row;
        const int teams = static_cast<int>(rows < c.teams ? rows : c.teams);
        for (int k = threadIdx.x; k < c.cols * GROUP; k += blockDim.x) {
            const int64_t channel = p.channel - (threadIdx.x % c.cols) * GROUP + k;
            if (channel >= c.C)
                continue;
            float mean = 0.f, m2 = 0.f, sum = 0.f;
            for (int w = 0; w < teams; ++w) {
                const float count = static_cast<float>((rows - w + c.teams - 1) / c.teams);
                sum = fmaf(count, lds[w * c.cols * GROUP + k].a - lds[k].a, sum);
            }
            mean = lds[k].a + sum / static_cast<float>(rows);
            for (int w = 0; w < teams; ++w) {
                const float count = static_cast<float>((rows - w + c.teams - 1) / c.teams);
                const Pair q = lds[w * c.cols * GROUP + k];
                m2 += fmaf(count * (q.a - mean), q.a - mean, q.b);
            }
            *pair_at(partial, c, p.n, p.chunk, channel) = Pair{mean, m2};
        }
        __syncthreads();
    }
}

__device__ __forceinline__ double workgroup_sum(double v, double* lds)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (unsigned i = 0; i < blockDim.x / 64; ++i)
        v += lds[i];
    return v;
}

// Each group's mean and rstd, one workgroup a group.
__global__ __launch_bounds__(SUM_THREADS) void group_stats_kernel(const Pair* __restrict__ partial, Cut c, float eps,
                                                                  float* __restrict__ mean_out,
                                                                  float* __restrict__ rstd_out)
{
    __shared__ double lds[SUM_THREADS / 64];
    const int64_t pairs = c.chunks * c.D;
    const double count = static_cast<double>(c.L) * static_cast<double>(c.D);
    for (int64_t q = blockIdx.x; q < c.N * c.groups; q += gridDim.x) {
        const int64_t n = q / c.groups, first = (q - n * c.groups) * c.D;
        auto at = [&](int64_t i, double& rows) {
            const int64_t chunk = i / c.D;
            rows = static_cast<double>(chunk + 1 < c.chunks ? c.rows : c.L - chunk * c.rows);
            return partial[(n * c.chunks + chunk) * c.C + first + (i - chunk * c.D)];
        };
        double s = 0.0, rows;
        for (int64_t i = threadIdx.x; i < pairs; i += SUM_THREADS) {
            const Pair p = at(i, rows);
            s += rows * p.a;
        }
        const double mean = workgroup_sum(s, lds) / count;
        s = 0.0;
        for (int64_t i = threadIdx.x; i < pairs; i += SUM_THREADS) {
            const Pair p = at(i, rows);
            s += p.b + rows * (p.a - mean) * (p.a - mean);
        }
        s = workgroup_sum(s, lds);
        if (threadIdx.x == 0) {
            mean_out[q] = static_cast<float>(mean);
            rstd_out[q] = static_cast<float>(1.0 / sqrt(s / count + eps));
        }
    }
}

// 1 / (1 + e^-z)
__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float activated(float z)
{
    if (ACT == POSEIDON_ACT_RELU)
        return z > 0.f || z != z ? z : 0.f;
    if (ACT == POSEIDON_ACT_SILU)
        return z * sigmoid(z);
    return z;
}

template <typename T, int ACT>
__global__ __launch_bounds__(MOST_THREADS) void forward_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                               const float* __restrict__ beta, Cut c, int64_t work,
                                                               const float* __restrict__ mean_in,
                                                               const float* __restrict__ rstd_in, T* __restrict__ y)
{
    for (int64_t b = blockIdx.x; b < work; b += gridDim.x) {
        const Place p = place_of(c, b);
        if (!p.active)
            continue;
        const int64_t left = c.C - p.channel;
        float mean[GROUP], scale[GROUP], shift[GROUP], v[GROUP];
        per_channel(mean_in, c, p.n, p.channel, mean);
        per_channel(rstd_in, c, p.n, p.channel, scale);
        load_some(gamma + p.channel, left, v);
        load_some(beta + p.channel, left, shift);
#pragma unroll
        for (int i = 0; i < GROUP; ++i)
            scale[i] *= v[i];
        for (int64_t r = p.first_row + p.team; r < p.end_row; r += c.teams) {
            const int64_t at = (p.n * c.L + r) * c.C + p.channel;
            load_some(x + at, left, v);
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] = activated<ACT>(fmaf(v[i] - mean[i], scale[i], shift[i]));
            store_some(y + at, left, v);
        }
    }
}

// ---------------------------------------------------------------------------
// Backward: dz = dy act'(z), with n = (x - mean) rstd and z = n gamma + beta.
// ---------------------------------------------------------------------------
// The gradient that reaches z.  ReLU: z next to 0 -- within 2^-20 of its terms,
// which fp32 gets right to 2^-22 -- is made again in 64 bits, so that which side
// it falls on does not depend on how it is rounded.
template <int ACT>
__device__ __forceinline__ float gradient(float dy, float x, float mean, float rstd, float n, float gamma, float beta)
{
    if (ACT == POSEIDON_ACT_NONE)
        return dy;
    const float z = fmaf(n, gamma, beta);
    if (ACT == POSEIDON_ACT_SILU) {
        const float q = sigmoid(z);
        return dy * q * fmaf(z, 1.f - q, 1.f);
    }
    bool on = z > 0.f;
    if (fabsf(z) <= 0x1p-20f * (fabsf(n * gamma) + fabsf(beta)))
        on = (static_cast<double>(x) - mean) * rstd * gamma + beta > 0.0;
    return on ? dy : 0.f;
}

// Sums over each chunk's rows: dz and dz n of each channel.
template <typename T, int ACT>
__global__ __launch_bounds__(MOST_THREADS) void chunk_sums_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
    Cut c, int64_t work, const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
    Pair* __restrict__ partial)
{
    __shared__ Pair lds[MOST_THREADS * GROUP];
    for (int64_t b = blockIdx.x; b < work; b += gridDim.x) {
        const Place p = place_of(c, b);
        const int64_t left = c.C - p.channel;
        float s1[GROUP] = {}, s2[GROUP] = {};
        if (p.active) {
            float mean[GROUP], rstd[GROUP], w[GROUP], shift[GROUP], v[GROUP], d[GROUP];
            per_channel(mean_in, c, p.n, p.channel, mean);
            per_channel(rstd_in, c, p.n, p.channel, rstd);
            load_some(gamma + p.channel, left, w);
            load_some(beta + p.channel, left, shift);
            for (int64_t r = p.first_row + p.team; r < p.end_row; r += c.teams) {
                const int64_t at = (p.n * c.L + r) * c.C + p.channel;
                load_some(x + at, left, v);
                load_some(dy + at, left, d);
#pragma unroll
                for (int i = 0; i < GROUP; ++i) {
                    const float n = (v[i] - mean[i]) * rstd[i];
                    const float dz = gradient<ACT>(d[i], v[i], mean[i], rstd[i], n, w[i], shift[i]);
                    s1[i] += dz;
                    s2[i] = fmaf(dz, n, s2[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                lds[threadIdx.x * GROUP + i] = Pair{s1[i], s2[i]};
        }
        __syncthreads();
        for (int k = threadIdx.x; k < c.cols * GROUP; k += blockDim.x) {
            const int64_t channel = p.channel - (threadIdx.x % c.cols) * GROUP + k;
            if (channel >= c.C)
                continue;
            Pair s{0.f, 0.f};
            for (int w = 0; w < c.teams; ++w) {
                s.a += lds[w * c.cols * GROUP + k].a;
                s.b += lds[w * c.cols * GROUP + k].b;
            }
            *pair_at(partial, c, p.n, p.chunk, channel) = s;
        }
        __syncthreads();
    }
}

// Each group's averages of g = gamma dz and of g n (the first N groups of work),
// then dgamma and dbeta, SUM_COLS channels a workgroup.
constexpr int SUM_COLS = 16;

__global__ __launch_bounds__(SUM_THREADS) void join_sums_kernel(const Pair* __restrict__ partial, Cut c,
                                                                const float* __restrict__ gamma,
                                                                Pair* __restrict__ averages,
                                                                float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ double lds[SUM_THREADS * 2];
    const int64_t of_groups = c.N * c.groups, work = of_groups + (c.C + SUM_COLS - 1) / SUM_COLS;
    const int64_t pairs = c.chunks * c.D;
    const double count = static_cast<double>(c.L) * static_cast<double>(c.D);
    for (int64_t q = blockIdx.x; q < work; q += gridDim.x) {
        if (q < of_groups) {
            const int64_t n = q / c.groups, first = (q - n * c.groups) * c.D;
            double s1 = 0.0, s2 = 0.0;
            for (int64_t i = threadIdx.x; i < pairs; i += SUM_THREADS) {
                const int64_t chunk = i / c.D, channel = first + (i - chunk * c.D);
                const Pair p = partial[(n * c.chunks + chunk) * c.C + channel];
                s1 += static_cast<double>(gamma[channel]) * p.a;
                s2 += static_cast<double>(gamma[channel]) * p.b;
            }
            s1 = workgroup_sum(s1, lds);
            s2 = workgroup_sum(s2, lds);
            if (threadIdx.x == 0)
                averages[q] = Pair{static_cast<float>(s1 / count), static_cast<float>(s2 / count)};
            continue;
        }
        constexpr int SLICES = SUM_THREADS / SUM_COLS;
        const int lane = threadIdx.x % SUM_COLS, w = threadIdx.x / SUM_COLS;
        const int64_t channel = (q - of_groups) * SUM_COLS + lane;
        double s1 = 0.0, s2 = 0.0;
        if (channel < c.C)
            for (int64_t i = w; i < c.N * c.chunks; i += SLICES) {
                const Pair p = partial[i * c.C + channel];
                s1 += p.a;
                s2 += p.b;
            }
        __syncthreads();
        lds[threadIdx.x * 2] = s1;
        lds[threadIdx.x * 2 + 1] = s2;
        __syncthreads();
        if (w == 0 && channel < c.C) {
            s1 = s2 = 0.0;
            for (int i = 0; i < SLICES; ++i) {
                s1 += lds[(i * SUM_COLS + lane) * 2];
                s2 += lds[(i * SUM_COLS + lane) * 2 + 1];
            }
            dbeta[channel] = static_cast<float>(s1);
            dgamma[channel] = static_cast<float>(s2);
        }
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(MOST_THREADS) void backward_kernel(
    const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
    Cut c, int64_t work, const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
    const Pair* __restrict__ averages, T* __restrict__ dx)
{
    for (int64_t b = blockIdx.x; b < work; b += gridDim.x) {
        const Place p = place_of(c, b);
        if (!p.active)
            continue;
        const int64_t left = c.C - p.channel;
        float mean[GROUP], rstd[GROUP], w[GROUP], shift[GROUP], a1[GROUP], a2[GROUP], v[GROUP], d[GROUP];
        per_channel(mean_in, c, p.n, p.channel, mean);
        per_channel(rstd_in, c, p.n, p.channel, rstd);
        load_some(gamma + p.channel, left, w);
        load_some(beta + p.channel, left, shift);
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            const Pair q = p.channel + i < c.C ? averages[p.n * c.groups + (p.channel + i) / c.D] : Pair{0.f, 0.f};
            a1[i] = q.a;
            a2[i] = q.b;
        }
        for (int64_t r = p.first_row + p.team; r < p.end_row; r += c.teams) {
            const int64_t at = (p.n * c.L + r) * c.C + p.channel;
            load_some(x + at, left, v);
            load_some(dy + at, left, d);
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const float n = (v[i] - mean[i]) * rstd[i];
                const float dz = gradient<ACT>(d[i], v[i], mean[i], rstd[i], n, w[i], shift[i]);
                v[i] = rstd[i] * (fmaf(w[i], dz, -a1[i]) - n * a2[i]);
            }
            store_some(dx + at, left, v);
        }
    }
}

// ---------------------------------------------------------------------------
// Launches.
// ---------------------------------------------------------------------------
int64_t workgroups(const Cut& c) { return c.N * c.chunks * c.sides; }

// Within a launch's limit of 2^32 threads: the kernels walk what is over.
unsigned grid_for(int64_t work) { return static_cast<unsigned>(std::min<int64_t>(work, 1 << 20)); }

int64_t partial_bytes(const Cut& c) { return c.N * c.chunks * c.C * static_cast<int64_t>(sizeof(Pair)); }

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
hipError_t forward_typed(const Cut& c, const T* x, const float* gamma, const float* beta, float eps, int32_t act, T* y,
                         float* mean, float* rstd, void* ws, hipStream_t s)
{
    const int64_t work = workgroups(c);
    Pair* partial = static_cast<Pair*>(ws);
    chunk_stats_kernel<T><<<grid_for(work), c.threads, 0, s>>>(x, c, work, partial);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess)
        return rc;
    group_stats_kernel<<<grid_for(c.N * c.groups), SUM_THREADS, 0, s>>>(partial, c, eps, mean, rstd);
    rc = hipGetLastError();
    if (rc != hipSuccess)
        return rc;
    with_act(act, [&](auto a) {
        forward_kernel<T, decltype(a)::value><<<grid_for(work), c.threads, 0, s>>>(x, gamma, beta, c, work, mean, rstd,
                                                                                   y);
    });
    return hipGetLastError();
}

template <typename T>
hipError_t backward_typed(const Cut& c, const T* dy, const T* x, const float* gamma, const float* beta,
                          const float* mean, const float* rstd, int32_t act, T* dx, float* dgamma, float* dbeta,
                          void* ws, hipStream_t s)
{
    const int64_t work = workgroups(c);
    Pair* partial = static_cast<Pair*>(ws);
    Pair* averages = partial + c.N * c.chunks * c.C;
    hipError_t rc = hipSuccess;
    if (work > 0) {
        with_act(act, [&](auto a) {
            chunk_sums_kernel<T, decltype(a)::value><<<grid_for(work), c.threads, 0, s>>>(dy, x, gamma, beta, c, work,
                                                                                          mean, rstd, partial);
        });
        rc = hipGetLastError();
        if (rc != hipSuccess)
            return rc;
    }
    join_sums_kernel<<<grid_for(c.N * c.groups + ceil_div(c.C, SUM_COLS)), SUM_THREADS, 0, s>>>(partial, c, gamma,
                                                                                                 averages, dgamma,
                                                                                                 dbeta);
    rc = hipGetLastError();
    if (rc != hipSuccess || work == 0)
        return rc;
    with_act(act, [&](auto a) {
        backward_kernel<T, decltype(a)::value><<<grid_for(work), c.threads, 0, s>>>(dy, x, gamma, beta, c, work, mean,
                                                                                    rstd, averages, dx);
    });
    return hipGetLastError();
}

}  // namespace

int64_t group_norm_workspace(int32_t op, int64_t N, int64_t L, int64_t C, int64_t groups, int32_t)
{
    const Cut c = make_cut(N, L, C, groups);
    return partial_bytes(c) + (op == POSEIDON_GROUP_NORM_BACKWARD ? N * groups * static_cast<int64_t>(sizeof(Pair)) : 0);
}

hipError_t launch_group_norm_forward(const void* x, const float* gamma, const float* beta, int64_t N, int64_t L,
                                     int64_t C, int64_t groups, int32_t dtype, float eps, int32_t act, void* y,
                                     float* mean, float* rstd, void* ws, hipStream_t stream)
{
    const Cut c = make_cut(N, L, C, groups);
    if (dtype == POSEIDON_BF16)
        return forward_typed(c, static_cast<const __bf16*>(x), gamma, beta, eps, act, static_cast<__bf16*>(y), mean,
                             rstd, ws, stream);
    return forward_typed(c, static_cast<const float*>(x), gamma, beta, eps, act, static_cast<float*>(y), mean, rstd,
                         ws, stream);
}

hipError_t launch_group_norm_backward(const void* dy, const void* x, const float* gamma, const float* beta,
                                      const float* mean, const float* rstd, int64_t N, int64_t L, int64_t C,
                                      int64_t groups, int32_t dtype, int32_t act, void* dx, float* dgamma,
                                      float* dbeta, void* ws, hipStream_t stream)
{
    const Cut c = make_cut(N, L, C, groups);
    if (dtype == POSEIDON_BF16)
        return backward_typed(c, static_cast<const __bf16*>(dy), static_cast<const __bf16*>(x), gamma, beta, mean,
                              rstd, act, static_cast<__bf16*>(dx), dgamma, dbeta, ws, stream);
    return backward_typed(c, static_cast<const float*>(dy), static_cast<const float*>(x), gamma, beta, mean, rstd,
                          act, static_cast<float*>(dx), dgamma, dbeta, ws, stream);
}

}  // namespace poseidon
