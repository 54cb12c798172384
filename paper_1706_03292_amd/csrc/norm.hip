// Layer norm with residual and dropout in the same pass, its backward pass,
// and dropout alone (include/poseidon.h gives the formulas).  All of it is a
// few operations per value, bound by memory: what counts is that every input
// is read once, every output written once, and that enough loads are in
// flight.  With residual and dropout, bf16: forward 16384 x 4096 112 us (4.8 TB/s;
// a device copy reaches 5.2), backward 16384 x 2048 73 us (4.6 TB/s), dropout
// alone 8191 x 4096 38 us (5.3 TB/s).
//
// A row is held in registers by a team of threads (16, 64, 256 or 1024: the
// fewest that leave a thread at most four groups of eight neighbours), so mean
// and variance take two passes over registers, not over memory, in fp32.  Rows
// longer than 32768 values are read three times instead.
//
// The backward pass gives each thread the same columns for all the rows its
// team walks, so dgamma and dbeta are sums in registers; the teams of a
// workgroup add theirs through LDS in a fixed order, each workgroup writes one
// partial row, and a second kernel adds the partials in a fixed order too:
// the result does not depend on timing.
#include "elements.h"

namespace poseidon {
namespace {

constexpr int THREADS = 256;

struct Drop {
    const uint64_t* rng;   // seed, offset (device memory); unread when thr = 0
    uint32_t thr;
    float scale;
};

__device__ __forceinline__ Rng read_rng(const Drop& d) { return d.thr ? Rng{d.rng[0], d.rng[1]} : Rng{0, 0}; }

// ---------------------------------------------------------------------------
// Dropout alone: y = (residual +) keep * x / (1 - p), one group a thread.
// PLAIN: the rows' groups are the flat array's (one row, or rows of a multiple
// of eight), so a group's place needs no division.
// ---------------------------------------------------------------------------
template <typename T, bool RES, bool PLAIN>
__global__ __launch_bounds__(THREADS) void dropout_kernel(const T* __restrict__ x, const T* __restrict__ res,
                                                          int64_t groups, int64_t per_row, int64_t cols, Drop d,
                                                          T* __restrict__ y)
{
    const Rng r = read_rng(d);
    const int64_t step = static_cast<int64_t>(gridDim.x) * THREADS;
    for (int64_t g = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; g < groups; g += step) {
        int64_t at = g * GROUP, left = cols % GROUP == 0 ? GROUP : cols - at;
        if (!PLAIN) {
            const int64_t row = g / per_row, c = (g - row * per_row) * GROUP;
            at = row * cols + c;
            left = cols - c;
        }
        float v[GROUP], q[GROUP];
        load_some(x + at, left, v);
        if (RES)
            load_some(res + at, left, q);
        if (d.thr)
            drop_group(v, r, static_cast<uint64_t>(g), d.thr, d.scale);
        if (RES)
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] += q[i];
        store_some(y + at, left, v);
    }
}

// ---------------------------------------------------------------------------
// Sums over a team of TPR threads (a power of two; more than 64: the whole
// workgroup, through LDS).
// ---------------------------------------------------------------------------
// (lds: a place per wave)
template <int TPR>
__device__ __forceinline__ float team_sum(float v, float* lds)
{
#pragma unroll
    for (int m = 1; m < (TPR < 64 ? TPR : 64); m <<= 1)
        v += __shfl_xor(v, m);
    if constexpr (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w)
            v += lds[w];
    }
    return v;
}

template <typename T, int TPR, int NG>
__global__ __launch_bounds__(TPR > THREADS ? TPR : THREADS) void norm_forward_kernel(
    const T* __restrict__ x, const T* __restrict__ res, const float* __restrict__ gamma,
    const float* __restrict__ beta, int64_t rows, int64_t cols, float eps, Drop d, T* __restrict__ h,
    T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int NT = TPR > THREADS ? TPR : THREADS, TEAMS = NT / TPR;
    __shared__ float lds[16];
    const int t = threadIdx.x % TPR;
    const int64_t per_row = (cols + GROUP - 1) / GROUP;
    const Rng r = read_rng(d);
    // A team above 64 threads is the workgroup: it meets the barriers together.
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * TEAMS + threadIdx.x / TPR; row < rows;
         row += static_cast<int64_t>(gridDim.x) * TEAMS) {
        const int64_t base = row * cols;
        float v[NG][GROUP];
    #pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t g = t + static_cast<int64_t>(i) * TPR;
            load_some(x + base + g * GROUP, cols - g * GROUP, v[i]);
        }
        if (res) {
            float q[NG][GROUP];
    #pragma unroll
            for (int i = 0; i < NG; ++i) {
                const int64_t g = t + static_cast<int64_t>(i) * TPR;
                load_some(res + base + g * GROUP, cols - g * GROUP, q[i]);
            }
    #pragma unroll
            for (int i = 0; i < NG; ++i) {
                const int64_t g = t + static_cast<int64_t>(i) * TPR;
                if (d.thr && g < per_row)
                    drop_group(v[i], r, static_cast<uint64_t>(row * per_row + g), d.thr, d.scale);
    #pragma unroll
                for (int e = 0; e < GROUP; ++e)
                    v[i][e] += q[i][e];
            }
        } else if (d.thr) {
    #pragma unroll
            for (int i = 0; i < NG; ++i) {
                const int64_t g = t + static_cast<int64_t>(i) * TPR;
                if (g < per_row)
                    drop_group(v[i], r, static_cast<uint64_t>(row * per_row + g), d.thr, d.scale);
            }
        }
        float s = 0.f;
    #pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t g = t + static_cast<int64_t>(i) * TPR;
            if (h && g < per_row)
                store_some(h + base + g * GROUP, cols - g * GROUP, v[i]);
    #pragma unroll
            for (int e = 0; e < GROUP; ++e)
                s += v[i][e];   // past the row's end: 0 (load_some; a dropped 0 stays 0)
        }
        const float mean = team_sum<TPR>(s, lds) / static_cast<float>(cols);
        s = 0.f;
    #pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t left = cols - (t + static_cast<int64_t>(i) * TPR) * GROUP;
    #pragma unroll
            for (int e = 0; e < GROUP; ++e) {
                v[i][e] -= mean;
                s = fmaf(e < left ? v[i][e] : 0.f, v[i][e], s);
            }
        }
        const float rstd = 1.f / sqrtf(team_sum<TPR>(s, lds) / static_cast<float>(cols) + eps);
    #pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t g = t + static_cast<int64_t>(i) * TPR, left = cols - g * GROUP;
            if (g < per_row) {
                float a[GROUP], b[GROUP];
                load_some(gamma + g * GROUP, left, a);
                load_some(beta + g * GROUP, left, b);
    #pragma unroll
                for (int e = 0; e < GROUP; ++e)
                    v[i][e] = fmaf(v[i][e] * rstd, a[e], b[e]);
                store_some(y + base + g * GROUP, left, v[i]);
            }
        }
        if (t == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
    }
}

// Rows too long for registers: one workgroup a row, the row's values made
// again in each of three passes (mean, variance, result).
constexpr int LONG_THREADS = 1024;

template <typename T>
__device__ __forceinline__ void row_group(const T* x, const T* res, int64_t base, int64_t row, int64_t per_row,
                                          int64_t cols, int64_t g, const Drop& d, const Rng& r, float (&v)[GROUP])
{
    load_some(x + base + g * GROUP, cols - g * GROUP, v);
    if (d.thr)
        drop_group(v, r, static_cast<uint64_t>(row * per_row + g), d.thr, d.scale);
    if (res) {
        float q[GROUP];
        load_some(res + base + g * GROUP, cols - g * GROUP, q);
#pragma unroll
        for (int e = 0; e < GROUP; ++e)
            v[e] += q[e];
    }
}

template <typename T>
__global__ __launch_bounds__(LONG_THREADS) void norm_forward_long(
    const T* __restrict__ x, const T* __restrict__ res, const float* __restrict__ gamma,
    const float* __restrict__ beta, int64_t rows, int64_t cols, float eps, Drop d, T* __restrict__ h,
    T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    __shared__ float lds[16];
    const int64_t per_row = (cols + GROUP - 1) / GROUP;
    const Rng r = read_rng(d);
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t base = row * cols;
        float v[GROUP], s = 0.f;
        for (int64_t g = threadIdx.x; g < per_row; g += LONG_THREADS) {
            row_group(x, res, base, row, per_row, cols, g, d, r, v);
            if (h)
                store_some(h + base + g * GROUP, cols - g * GROUP, v);
    #pragma unroll
            for (int e = 0; e < GROUP; ++e)
                s += v[e];
        }
        const float mean = team_sum<LONG_THREADS>(s, lds) / static_cast<float>(cols);
        s = 0.f;
        for (int64_t g = threadIdx.x; g < per_row; g += LONG_THREADS) {
            row_group(x, res, base, row, per_row, cols, g, d, r, v);
    #pragma unroll
            for (int e = 0; e < GROUP; ++e) {
                const float c = e < cols - g * GROUP ? v[e] - mean : 0.f;
                s = fmaf(c, c, s);
            }
        }
        const float rstd = 1.f / sqrtf(team_sum<LONG_THREADS>(s, lds) / static_cast<float>(cols) + eps);
        for (int64_t g = threadIdx.x; g < per_row; g += LONG_THREADS) {
            row_group(x, res, base, row, per_row, cols, g, d, r, v);
            float a[GROUP], b[GROUP];
            load_some(gamma + g * GROUP, cols - g * GROUP, a);
            load_some(beta + g * GROUP, cols - g * GROUP, b);
    #pragma unroll
            for (int e = 0; e < GROUP; ++e)
                v[e] = fmaf((v[e] - mean) * rstd, a[e], b[e]);
            store_some(y + base + g * GROUP, cols - g * GROUP, v);
        }
        if (threadIdx.x == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
    }
}

// ---------------------------------------------------------------------------
// Backward: with g = dy * gamma and n = (h - mean) * rstd,
//   dh = rstd * (g - avg(g) - n * avg(g * n)) + dres,   dx = dropout(dh),
//   dgamma = sum over rows of dy * n,                   dbeta = sum over rows of dy.
// ---------------------------------------------------------------------------
// Where a workgroup's sums over its rows go, `stride` values apart: partial
// rows, or (one workgroup) the results themselves.
struct WeightSums {
    float* dgamma;
    float* dbeta;
    int64_t stride;
};

template <typename T, int TPR, int NG>
__global__ __launch_bounds__(TPR > THREADS ? TPR : THREADS) void norm_backward_kernel(
    const T* __restrict__ dy, const T* __restrict__ h, const float* __restrict__ gamma,
    const float* __restrict__ mean_in, const float* __restrict__ rstd_in, const T* __restrict__ dres, int64_t rows,
    int64_t cols, Drop d, T* __restrict__ dx, T* __restrict__ dh, WeightSums out)
{
    constexpr int NT = TPR > THREADS ? TPR : THREADS, TEAMS = NT / TPR;
    __shared__ float lds[32];
    __shared__ float sums[TEAMS > 1 ? 2 * TPR * NG * GROUP : 1];
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR;
    const int64_t per_row = (cols + GROUP - 1) / GROUP, step = static_cast<int64_t>(gridDim.x) * TEAMS;
    const float inv = 1.f / static_cast<float>(cols);
    const Rng r = read_rng(d);
    float dg[NG][GROUP] = {}, db[NG][GROUP] = {};
    // The next row's values are on their way while a row is worked on: a team
    // has one row at a time, and its sums would otherwise wait for each row's
    // loads in full (16384 x 2048 bf16 with residual and dropout: 100 us so).
    Raw<T> ry[NG], rh[NG], re[NG];
    float mean = 0.f, rstd = 0.f;
    auto fetch = [&](int64_t row) {
        const int64_t base = row * cols;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t c = (t + static_cast<int64_t>(i) * TPR) * GROUP;
            load_raw(dy + base + c, cols - c, ry[i]);
            load_raw(h + base + c, cols - c, rh[i]);
            if (dres)
                load_raw(dres + base + c, cols - c, re[i]);
        }
        mean = mean_in[row];
        rstd = rstd_in[row];
    };
    int64_t row = static_cast<int64_t>(blockIdx.x) * TEAMS + team;
    if (row < rows)
        fetch(row);
    // A team above 64 threads is the workgroup: it meets the sums' barriers
    // together.
    for (; row < rows; row += step) {
        const int64_t base = row * cols;
        float g[NG][GROUP], n[NG][GROUP];
        Raw<T> e[NG];
        const float rs = rstd;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            e[i] = re[i];
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                g[i][k] = raw_value(ry[i], k);   // past the row's end: 0, and nothing is stored
                n[i][k] = (raw_value(rh[i], k) - mean) * rs;
            }
        }
        if (row + step < rows)
            fetch(row + step);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t c = (t + static_cast<int64_t>(i) * TPR) * GROUP;
            float a[GROUP];
            load_some(gamma + c, cols - c, a);
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                dg[i][k] = fmaf(g[i][k], n[i][k], dg[i][k]);
                db[i][k] += g[i][k];
                g[i][k] *= a[k];
                s1 += g[i][k];
                s2 = fmaf(g[i][k], n[i][k], s2);
            }
        }
        s1 = team_sum<TPR>(s1, lds) * inv;
        s2 = team_sum<TPR>(s2, lds + 16) * inv;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int64_t q = t + static_cast<int64_t>(i) * TPR, c = q * GROUP;
            if (q < per_row) {
#pragma unroll
                for (int k = 0; k < GROUP; ++k) {
                    const float v = rs * (g[i][k] - s1 - n[i][k] * s2);
                    g[i][k] = dres ? v + raw_value(e[i], k) : v;
                }
                store_some(dh + base + c, cols - c, g[i]);
                if (d.thr) {
                    drop_group(g[i], r, static_cast<uint64_t>(row * per_row + q), d.thr, d.scale);
                    store_some(dx + base + c, cols - c, g[i]);
                }
            }
        }
    }
    // The workgroup's sums: its teams in order.
    if constexpr (TEAMS > 1) {
        for (int w = 0; w < TEAMS; ++w) {
            if (team == w) {
#pragma unroll
                for (int i = 0; i < NG; ++i)
#pragma unroll
                    for (int k = 0; k < GROUP; ++k) {
                        float* a = sums + ((i * GROUP + k) * TPR + t) * 2;
                        if (w > 0) {
                            dg[i][k] += a[0];
                            db[i][k] += a[1];
                        }
                        if (w + 1 < TEAMS) {
                            a[0] = dg[i][k];
                            a[1] = db[i][k];
                        }
                    }
            }
            __syncthreads();
        }
        if (team != TEAMS - 1)
            return;
    }
    const int64_t part = static_cast<int64_t>(blockIdx.x) * out.stride;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        const int64_t c = (t + static_cast<int64_t>(i) * TPR) * GROUP;
        if (c < cols) {
            store_some(out.dgamma + part + c, cols - c, dg[i]);
            store_some(out.dbeta + part + c, cols - c, db[i]);
        }
    }
}

// Rows too long for registers: one workgroup walks whole rows (two passes
// over each for the averages and the result), and dgamma and dbeta are left
// to a kernel of their own.
template <typename T>
__global__ __launch_bounds__(LONG_THREADS) void norm_backward_long(
    const T* __restrict__ dy, const T* __restrict__ h, const float* __restrict__ gamma,
    const float* __restrict__ mean_in, const float* __restrict__ rstd_in, const T* __restrict__ dres, int64_t rows,
    int64_t cols, Drop d, T* __restrict__ dx, T* __restrict__ dh)
{
    __shared__ float lds[32];
    const int64_t per_row = (cols + GROUP - 1) / GROUP;
    const Rng r = read_rng(d);
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t base = row * cols;
        const float mean = mean_in[row], rstd = rstd_in[row];
        float g[GROUP], n[GROUP], a[GROUP], s1 = 0.f, s2 = 0.f;
        for (int64_t q = threadIdx.x; q < per_row; q += LONG_THREADS) {
            const int64_t c = q * GROUP;
            load_some(dy + base + c, cols - c, g);
            load_some(h + base + c, cols - c, n);
            load_some(gamma + c, cols - c, a);
    #pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                g[k] *= a[k];
                s1 += g[k];
                s2 = fmaf(g[k], (n[k] - mean) * rstd, s2);
            }
        }
        s1 = team_sum<LONG_THREADS>(s1, lds) / static_cast<float>(cols);
        s2 = team_sum<LONG_THREADS>(s2, lds + 16) / static_cast<float>(cols);
        for (int64_t q = threadIdx.x; q < per_row; q += LONG_THREADS) {
            const int64_t c = q * GROUP;
            load_some(dy + base + c, cols - c, g);
            load_some(h + base + c, cols - c, n);
            load_some(gamma + c, cols - c, a);
    #pragma unroll
            for (int k = 0; k < GROUP; ++k)
                g[k] = rstd * (g[k] * a[k] - s1 - (n[k] - mean) * rstd * s2);
            if (dres) {
                load_some(dres + base + c, cols - c, a);
    #pragma unroll
                for (int k = 0; k < GROUP; ++k)
                    g[k] += a[k];
            }
            store_some(dh + base + c, cols - c, g);
            if (d.thr) {
                drop_group(g, r, static_cast<uint64_t>(row * per_row + q), d.thr, d.scale);
                store_some(dx + base + c, cols - c, g);
            }
        }
    }
}

// Partial sums of dgamma and dbeta for long rows: a thread owns one group of
// columns, workgroup row y takes every gridDim.y-th row.
template <typename T>
__global__ __launch_bounds__(THREADS) void norm_weights_long(const T* __restrict__ dy, const T* __restrict__ h,
                                                             const float* __restrict__ mean_in,
                                                             const float* __restrict__ rstd_in, int64_t rows,
                                                             int64_t cols, WeightSums out)
{
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x) * GROUP;
    if (c >= cols)
        return;
    float dg[GROUP] = {}, db[GROUP] = {}, g[GROUP], n[GROUP];
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        load_some(dy + row * cols + c, cols - c, g);
        load_some(h + row * cols + c, cols - c, n);
        const float mean = mean_in[row], rstd = rstd_in[row];
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
            dg[k] = fmaf(g[k], (n[k] - mean) * rstd, dg[k]);
            db[k] += g[k];
        }
    }
    const int64_t part = static_cast<int64_t>(blockIdx.y) * out.stride;
    store_some(out.dgamma + part + c, cols - c, dg);
    store_some(out.dbeta + part + c, cols - c, db);
}

// dgamma and dbeta from `parts` partial rows: 16 columns a workgroup and turn, 16
// threads a column, each adding every 16th partial, then theirs in order.
constexpr int SUM_COLS = 16;

__global__ __launch_bounds__(THREADS) void norm_weights_kernel(const float* __restrict__ partial, int parts,
                                                               int64_t cols, float* __restrict__ dgamma,
                                                               float* __restrict__ dbeta)
{
    constexpr int SLICES = THREADS / SUM_COLS;
    __shared__ float lds[SLICES][SUM_COLS];
    const int lane = threadIdx.x % SUM_COLS, w = threadIdx.x / SUM_COLS;
    // (The whole workgroup takes each turn: it meets the barriers together.)
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * SUM_COLS; first < 2 * cols;
         first += static_cast<int64_t>(gridDim.x) * SUM_COLS) {
        const int64_t c = first + lane;
        float s = 0.f;
        if (c < 2 * cols)
#pragma unroll 16
            for (int p = w; p < parts; p += SLICES)
                s += partial[p * 2 * cols + c];
        lds[w][lane] = s;
        __syncthreads();
        if (w == 0 && c < 2 * cols) {
            s = 0.f;
#pragma unroll
            for (int i = 0; i < SLICES; ++i)
                s += lds[i][lane];
            if (c < cols)
                dgamma[c] = s;
            else
                dbeta[c - cols] = s;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Launches.
// ---------------------------------------------------------------------------
Drop make_drop(uint32_t thr, const int64_t* rng)
{
    // All dropped (thr = 65536): nothing is scaled.
    const float scale = thr >= 65536 ? 0.f : static_cast<float>(65536.0 / (65536.0 - thr));
    return Drop{reinterpret_cast<const uint64_t*>(rng), thr, scale};
}

constexpr int64_t LONGEST_FORWARD = 1024 * 4 * GROUP, LONGEST_BACKWARD = 512 * 2 * GROUP;   // values a team holds

// f(Int<TPR>, Int<NG>) for the team that holds a row of `cols` values.  The
// backward pass holds the row's three inputs, the next row's and two sums a
// column, so its threads take at most two groups (at four, with 290 registers,
// one wave a SIMD is left: 16384 x 2048 bf16 86 us, with one group of 256
// threads 68 us).
template <int V>
struct Int {
    static constexpr int value = V;
};

template <typename F>
hipError_t with_forward_team(int64_t cols, F&& f)
{
    const int64_t groups = (cols + GROUP - 1) / GROUP;
    if (groups <= 16)
        return f(Int<16>(), Int<1>());
    if (groups <= 64)
        return f(Int<64>(), Int<1>());
    if (groups <= 128)
        return f(Int<64>(), Int<2>());
    if (groups <= 256)
        return f(Int<64>(), Int<4>());
    if (groups <= 512)
        return f(Int<256>(), Int<2>());
    if (groups <= 1024)
        return f(Int<256>(), Int<4>());
    return f(Int<1024>(), Int<4>());
}

template <typename F>
hipError_t with_backward_team(int64_t cols, F&& f)
{
    const int64_t groups = (cols + GROUP - 1) / GROUP;
    if (groups <= 16)
        return f(Int<16>(), Int<1>());
    if (groups <= 64)
        return f(Int<64>(), Int<1>());
    if (groups <= 128)
        return f(Int<64>(), Int<2>());
    if (groups <= 256)
        return f(Int<256>(), Int<1>());
    if (groups <= 512)
        return f(Int<256>(), Int<2>());
    return f(Int<512>(), Int<2>());
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups for `work` workgroups' worth, within a launch's limit of 2^32
// threads: the kernels walk what is over.
unsigned grid_for(int64_t work) { return static_cast<unsigned>(std::min<int64_t>(work, 1 << 20)); }

// Workgroups of the backward pass: a few a CU keep its loads in flight, and
// each leaves one partial row.  One walks up to four rows a team by itself: its
// sums are the result, and the launch that adds partial rows is spared (a
// sixteen-row call is bound by its launches).
int backward_groups(int64_t rows, int64_t cols)
{
    const int64_t teams = cols > 1024 ? 1 : cols > 128 ? 4 : 16;
    if (rows <= 4 * teams)
        return 1;
    // Three a CU for the team of 256 threads with one group each, which needs the
    // fewest registers, two elsewhere.  16384 rows with residual and dropout, us
    // with two and three, bf16 then fp32: x 1032 74, 57 and 107, 90; x 1536 62, 52
    // and 97, 105; x 2048 78, 71 and 127, 136; outside that range x 1000 39, 36
    // and 71, 82; x 1024 34, 35 and 69, 78; x 2056 120, 99 and 158, 197; x 4096
    // 133, 142 and 260, 261; x 8192 274, 286 and 508, 527.
    const int64_t per_cu = cols > 1024 && cols <= 2048 ? 3 : 2;
    return static_cast<int>(std::min<int64_t>(ceil_div(rows, teams), per_cu * device_cu_count()));
}

template <typename T>
hipError_t dropout_typed(const T* x, const T* res, int64_t rows, int64_t cols, const Drop& d, T* y, hipStream_t s)
{
    const int64_t per_row = ceil_div(cols, GROUP), groups = rows * per_row;
    const unsigned grid = grid_for(ceil_div(groups, THREADS));
    const bool plain = cols % GROUP == 0 || rows == 1;
    auto* k = res ? (plain ? dropout_kernel<T, true, true> : dropout_kernel<T, true, false>)
                  : (plain ? dropout_kernel<T, false, true> : dropout_kernel<T, false, false>);
    k<<<grid, THREADS, 0, s>>>(x, res, groups, per_row, cols, d, y);
    return hipGetLastError();
}

template <typename T>
hipError_t forward_typed(const T* x, const T* res, const float* gamma, const float* beta, int64_t rows, int64_t cols,
                         float eps, const Drop& d, T* h, T* y, float* mean, float* rstd, hipStream_t s)
{
    if (cols > LONGEST_FORWARD) {
        norm_forward_long<T><<<grid_for(rows), LONG_THREADS, 0, s>>>(x, res, gamma, beta, rows, cols, eps, d, h, y,
                                                                     mean, rstd);
        return hipGetLastError();
    }
    return with_forward_team(cols, [&](auto tpr, auto ng) {
        constexpr int TPR = decltype(tpr)::value, NG = decltype(ng)::value, NT = TPR > THREADS ? TPR : THREADS;
        norm_forward_kernel<T, TPR, NG><<<grid_for(ceil_div(rows, NT / TPR)), NT, 0, s>>>(
            x, res, gamma, beta, rows, cols, eps, d, h, y, mean, rstd);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward_typed(const T* dy, const T* h, const float* gamma, const float* mean, const float* rstd,
                          const T* dres, int64_t rows, int64_t cols, const Drop& d, T* dx, T* dh, float* dgamma,
                          float* dbeta, float* partial, hipStream_t s)
{
    const int parts = backward_groups(rows, cols);
    const WeightSums sums = parts > 1 ? WeightSums{partial, partial + cols, 2 * cols} : WeightSums{dgamma, dbeta, 0};
    hipError_t rc = hipSuccess;
    if (cols > LONGEST_BACKWARD) {
        if (rows > 0)
            norm_backward_long<T><<<grid_for(rows), LONG_THREADS, 0, s>>>(dy, h, gamma, mean, rstd, dres, rows, cols, d,
                                                                          dx, dh);
        rc = hipGetLastError();
        if (rc != hipSuccess)
            return rc;
        const dim3 grid(static_cast<unsigned>(ceil_div(cols, THREADS * GROUP)), static_cast<unsigned>(parts));
        norm_weights_long<T><<<grid, THREADS, 0, s>>>(dy, h, mean, rstd, rows, cols, sums);
        rc = hipGetLastError();
    } else {
        rc = with_backward_team(cols, [&](auto tpr, auto ng) {
            constexpr int TPR = decltype(tpr)::value, NG = decltype(ng)::value, NT = TPR > THREADS ? TPR : THREADS;
            norm_backward_kernel<T, TPR, NG><<<static_cast<unsigned>(parts), NT, 0, s>>>(
                dy, h, gamma, mean, rstd, dres, rows, cols, d, dx, dh, sums);
            return hipGetLastError();
        });
    }
    if (rc != hipSuccess || parts == 1)
        return rc;
    norm_weights_kernel<<<grid_for(ceil_div(2 * cols, SUM_COLS)), THREADS, 0, s>>>(partial, parts, cols, dgamma,
                                                                                   dbeta);
    return hipGetLastError();
}

}  // namespace

int64_t norm_backward_workspace(int64_t rows, int64_t cols)
{
    return static_cast<int64_t>(backward_groups(rows, cols)) * 2 * cols * 4;
}

hipError_t launch_dropout(const void* x, const void* res, int64_t rows, int64_t cols, int32_t dtype, uint32_t thr,
                          const int64_t* rng, void* y, hipStream_t stream)
{
    const Drop d = make_drop(thr, rng);
    if (dtype == POSEIDON_BF16)
        return dropout_typed(static_cast<const __bf16*>(x), static_cast<const __bf16*>(res), rows, cols, d,
                             static_cast<__bf16*>(y), stream);
    return dropout_typed(static_cast<const float*>(x), static_cast<const float*>(res), rows, cols, d,
                         static_cast<float*>(y), stream);
}

hipError_t launch_norm_forward(const void* x, const void* res, const float* gamma, const float* beta, int64_t rows,
                               int64_t cols, int32_t dtype, float eps, uint32_t thr, const int64_t* rng, void* h,
                               void* y, float* mean, float* rstd, hipStream_t stream)
{
    const Drop d = make_drop(thr, rng);
    if (dtype == POSEIDON_BF16)
        return forward_typed(static_cast<const __bf16*>(x), static_cast<const __bf16*>(res), gamma, beta, rows, cols,
                             eps, d, static_cast<__bf16*>(h), static_cast<__bf16*>(y), mean, rstd, stream);
    return forward_typed(static_cast<const float*>(x), static_cast<const float*>(res), gamma, beta, rows, cols, eps,
                         d, static_cast<float*>(h), static_cast<float*>(y), mean, rstd, stream);
}

hipError_t launch_norm_backward(const void* dy, const void* h, const float* gamma, const float* mean,
                                const float* rstd, const void* dres, int64_t rows, int64_t cols, int32_t dtype,
                                uint32_t thr, const int64_t* rng, void* dx, void* dh, float* dgamma, float* dbeta,
                                void* workspace, hipStream_t stream)
{
    const Drop d = make_drop(thr, rng);
    float* partial = static_cast<float*>(workspace);
    if (dtype == POSEIDON_BF16)
        return backward_typed(static_cast<const __bf16*>(dy), static_cast<const __bf16*>(h), gamma, mean, rstd,
                              static_cast<const __bf16*>(dres), rows, cols, d, static_cast<__bf16*>(dx),
                              static_cast<__bf16*>(dh), dgamma, dbeta, partial, stream);
    return backward_typed(static_cast<const float*>(dy), static_cast<const float*>(h), gamma, mean, rstd,
                          static_cast<const float*>(dres), rows, cols, d, static_cast<float*>(dx),
                          static_cast<float*>(dh), dgamma, dbeta, partial, stream);
}

}  // namespace poseidon
