// Softmax cross entropy fused with the classifier's product (include/poseidon.h
// gives the formulas): T rows X (T x D), V classes W (V x D),
//
//     s = X W^T,  lse_t = log sum_v exp s_tv,  loss_t = lse_t - s_t,target
//     G = (exp(s - lse) - onehot(target)) * dloss,  dX = G W,  dW = G^T X.
//
// For many rows the logits never leave the matrix cores' registers: the forward
// tile's epilogue reduces its columns to a running maximum and sum per row, and a
// second kernel joins them; the backward pass makes the logits again, a piece of
// the vocabulary at a time, turns them into G in the epilogue and multiplies the
// piece with W and X.  The factor form, for layers that are synchronised by
// sufficient factors, writes G whole, because there G is the payload; up to 32
// rows take the forward pass too through memory.
//
// Bound: 2TVD operations a product on the matrix cores for many rows (8192 x
// 32768 x 2048 bf16: 0.89 ms, 1.2 PFLOP/s; backward 4097 x 50001 x 1024 2.6 ms,
// 512 x 21841 x 4096 fp32 1.54 ms), reading W for few (32 x 21841 x 4096 fp32: 85
// us, of which the product 75 at 4.7 TB/s; factors in bf16 101 us, W read twice).
#include <math.h>

#include "mfma_tile.h"

namespace poseidon {
namespace {

// exp(a - b).  The difference comes first: a product of a logit and log2 e would
// overflow where the logit is near the type's lowest value (a class that is to
// count for nothing), and its rounding error would grow with the logit.
__device__ __forceinline__ float exp_diff(float a, float b) { return __builtin_amdgcn_exp2f((a - b) * 1.44269504f); }

// A running maximum and the sum of exponentials below it.
struct Run {
    float m, s;
};

__device__ __forceinline__ Run join(Run a, Run b)
{
    const float m = fmaxf(a.m, b.m);
    // A side without a finite maximum (no column, or all -inf) adds nothing.
    const float ea = a.m == -INFINITY ? 0.f : exp_diff(a.m, m);
    const float eb = b.m == -INFINITY ? 0.f : exp_diff(b.m, m);
    return Run{m, fmaf(a.s, ea, b.s * eb)};
}

__device__ __forceinline__ float lse_of(Run r) { return r.m + logf(r.s); }

__device__ __forceinline__ bool counts(int64_t target, int64_t V) { return target >= 0 && target < V; }

// ---------------------------------------------------------------------------
// What a tile does with its sums.  acc[i][j][r] of lane l is row
// m0 + 16 i + l % 16, column n0 + 16 j + 4 (l / 16) + r.
// ---------------------------------------------------------------------------
enum Use { STATS, GRAD, STORE };

struct Out {
    // STATS: per row and column block the running maximum and sum, and the
    // target's logit.
    Run* part;
    int64_t nparts, block_first;
    float* target_logit;
    const int64_t* target;
    // GRAD: the piece's G from lse and dloss, in three bf16 parts (planes apart)
    // or fp32, columns v0 onwards of V.
    const float* lse;
    const float* dloss;
    void* g;
    int64_t ldg, g_plane;
    int64_t v0, V;
    // STORE: C (ldc apart), fp32 or bf16, added to what is there or not; with
    // several splits of k, split z's sums go to c + z * split_stride.
    void* c;
    int64_t ldc, split_stride;
    int32_t bf16, add;
};

typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4a __attribute__((ext_vector_type(4), aligned(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));

// One row's four neighbours at p (any boundary of their type), n of them.
__device__ __forceinline__ void put4(float* p, acc4 v, int n)
{
    if (n >= 4) {
        *reinterpret_cast<f4a*>(p) = v;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < n)
                p[r] = v[r];
    }
}

__device__ __forceinline__ void put4(__bf16* p, b4 v, int n)
{
    if (n >= 4) {
        *reinterpret_cast<b4a*>(p) = v;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < n)
                p[r] = v[r];
    }
}

// Two values rounded to bf16, the first in the low half; and what that leaves.
__device__ __forceinline__ unsigned bf16_pair(float a, float b)
{
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f2){a, b}, b2));
}
__device__ __forceinline__ f2 rest_of_pair(float a, float b, unsigned p)
{
    return f2{a - __builtin_bit_cast(float, p << 16), b - __builtin_bit_cast(float, p & 0xffff0000u)};
}

// STATS.  A row's maximum and the sum of exponentials below it over
// the wave's columns: in a lane first, then across the four lanes that share
// the row.
template <typename T, bool EDGE>
__device__ __forceinline__ void finish_stats(acc4 (&acc)[T::TM][T::TN], const Out& o, int64_t m0, int64_t n0,
                                             int64_t block, int rows, int cols, int wm, int wn, int lane)
{
    const int first = wn + 4 * (lane >> 4);   // the lane's columns: first + 16 j + r
    // What the rows need from memory is asked for at once: a wait per row
    // block was most of an epilogue's time.
    int64_t target[T::TM];
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int m = wm + 16 * i + (lane & 15);
        target[i] = m < rows ? o.target[m0 + m] : -1;
    }
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int m = wm + 16 * i + (lane & 15);
        const bool row = m < rows;
        const int64_t at = m0 + m;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!EDGE || first + 16 * j + r < cols)
                    top = fmaxf(top, acc[i][j][r]);
        // A NaN logit is no maximum, but makes the sum NaN.
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float from = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!EDGE || first + 16 * j + r < cols)
                    sum += exp_diff(acc[i][j][r], from);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (row) {
            if (lane < 16)
                o.part[at * o.nparts + block] = Run{top, sum};
            const int64_t t = target[i] - n0 - first;
            if (t >= 0 && t < T::WN) {
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (t == 16 * j + r && (!EDGE || first + 16 * j + r < cols))
                            o.target_logit[at] = acc[i][j][r];
            }
        }
    }
}

// GRAD.
template <typename T, bool EDGE>
__device__ __forceinline__ void finish_grad(acc4 (&acc)[T::TM][T::TN], const Out& o, int64_t m0, int64_t n0, int rows,
                                            int cols, int wm, int wn, int lane)
{
    // The lane's columns: first + STRIDE j + r.
    constexpr int STRIDE = T::SPREAD ? 4 : 16;
    const int first = wn + (T::SPREAD ? 16 : 4) * (lane >> 4);
    int64_t target[T::TM];
    float lses[T::TM], dlosses[T::TM];
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int m = wm + 16 * i + (lane & 15);
        const int64_t at = m0 + (m < rows ? m : 0);
        target[i] = o.target[at];
        lses[i] = o.lse[at];
        dlosses[i] = o.dloss[at];
    }
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int m = wm + 16 * i + (lane & 15);
        if (m >= rows)
            continue;
        const int64_t at = m0 + m, t = target[i];
        const bool has = counts(t, o.V);
        const float lse = has ? lses[i] : 0.f, d = has ? dlosses[i] : 0.f;
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float g = exp_diff(acc[i][j][r], lse) * d;
                // Rows without a target and, up to the row's end, past V: zeros.
                acc[i][j][r] = has && (!EDGE || first + STRIDE * j + r < cols) ? g : 0.f;
            }
        const int64_t tl = t - o.v0 - n0 - first;
        if (has && tl >= 0 && tl < T::WN) {
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (tl == STRIDE * j + r)
                        acc[i][j][r] -= d;
        }
        const int64_t to = at * o.ldg + n0 + first;
        // Runs of values that lie together (SPREAD: eight, else four).
        constexpr int RUN = T::SPREAD ? 2 : 1;
        typedef unsigned uw __attribute__((ext_vector_type(2 * RUN)));
#pragma unroll
        for (int j = 0; j < T::TN; j += RUN) {
            const bool in = !EDGE || n0 + first + STRIDE * j < o.ldg;   // ldg: a multiple of eight
            if constexpr (sizeof(typename T::M) == 4) {
                if (in)
                    *reinterpret_cast<acc4*>(static_cast<float*>(o.g) + to + STRIDE * j) = acc[i][j];
            } else {
                // bf16 parts: h and m rounded to nearest, l what is left, exactly.
                __bf16* g = static_cast<__bf16*>(o.g) + to + STRIDE * j;
                uw part[3];
#pragma unroll
                for (int q = 0; q < 2 * RUN; ++q) {
                    f2 x = {acc[i][j + q / 2][2 * (q % 2)], acc[i][j + q / 2][2 * (q % 2) + 1]};
                    part[0][q] = bf16_pair(x[0], x[1]);
                    x = rest_of_pair(x[0], x[1], part[0][q]);
                    part[1][q] = bf16_pair(x[0], x[1]);
                    x = rest_of_pair(x[0], x[1], part[1][q]);
                    part[2][q] = bf16_pair(x[0], x[1]);
                }
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (in)
                        *reinterpret_cast<uw*>(g + p * o.g_plane) = part[p];
            }
        }
    }
}

template <typename T, bool EDGE>
__device__ __forceinline__ void finish_store(acc4 (&acc)[T::TM][T::TN], const Out& o, int64_t m0, int64_t n0, int rows,
                                             int cols, int wm, int wn, int lane, int z)
{
    const int first = wn + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int m = wm + 16 * i + (lane & 15);
        if (m >= rows)
            continue;
        const int64_t at = m0 + m;
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            const int left = EDGE ? cols - first - 16 * j : 4;
            if (left <= 0)
                continue;
            acc4 v = acc[i][j];
            const int64_t to = at * o.ldc + n0 + first + 16 * j;
            if (o.bf16) {
                put4(static_cast<__bf16*>(o.c) + to, __builtin_convertvector(v, b4), left);
            } else {
                float* c = static_cast<float*>(o.c) + z * o.split_stride + to;
                if (o.add) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (r < left)
                            v[r] += c[r];
                }
                put4(c, v, left);
            }
        }
    }
}

template <typename T, Use USE>
__device__ __forceinline__ void finish(acc4 (&acc)[T::TM][T::TN], const Out& o, int64_t m0, int64_t n0, int64_t tile_n,
                                       int64_t M, int64_t N, int z)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int wm = (w / T::NWN) * T::WM, wn = (w % T::NWN) * T::WN;
    const int rows = static_cast<int>(M - m0 < T::BM ? M - m0 : T::BM);
    const int cols = static_cast<int>(N - n0 < T::BN ? N - n0 : T::BN);
    const bool edge = cols < T::BN;
    if constexpr (USE == STATS) {
        const int64_t block = o.block_first + tile_n * T::NWN + w % T::NWN;
        if (edge)
            finish_stats<T, true>(acc, o, m0, n0, block, rows, cols, wm, wn, lane);
        else
            finish_stats<T, false>(acc, o, m0, n0, block, rows, cols, wm, wn, lane);
    } else if constexpr (USE == GRAD) {
        if (edge)
            finish_grad<T, true>(acc, o, m0, n0, rows, cols, wm, wn, lane);
        else
            finish_grad<T, false>(acc, o, m0, n0, rows, cols, wm, wn, lane);
    } else {
        if (edge)
            finish_store<T, true>(acc, o, m0, n0, rows, cols, wm, wn, lane, z);
        else
            finish_store<T, false>(acc, o, m0, n0, rows, cols, wm, wn, lane, z);
    }
}

// A matrix copied with its rows padded to ldo values (zeros), rows without a
// target (where a target list is given) cleared.
struct RowCopy {
    const void* x;
    int64_t rows, cols, ldo;
    const int64_t* target;
    int64_t V;
    void* out;
};

template <typename E>
__device__ __forceinline__ void copy_rows(const RowCopy& o, int64_t first, int64_t step)
{
    const int64_t per_row = o.ldo / GROUP, groups = o.rows * per_row;
    for (int64_t q = first; q < groups; q += step) {
        const int64_t row = q / per_row, c = (q - row * per_row) * GROUP;
        float v[GROUP];
        load_some(static_cast<const E*>(o.x) + row * o.cols + c, o.cols - c, v);
        if (o.target && !counts(o.target[row], o.V))
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] = 0.f;
        store_group(static_cast<E*>(o.out) + row * o.ldo + c, v);
    }
}

// Rows m_first to M and columns n_first to N in tiles, over k split gridDim.y ways
// (k_split values each, a multiple of the step).  GRAD: workgroups past the tiles make the copy of X
// that dW's product reads, which would otherwise be a launch of its own.
template <typename T, Use USE>
__global__ __launch_bounds__(T::NT, 2) void product_kernel(Operand a, Operand b, Parts parts, Out o,
                                                           int64_t m_first, int64_t n_first, int64_t M, int64_t N,
                                                           int64_t K, int64_t k_split, int64_t tiles_m, int64_t tiles_n,
                                                           int group, RowCopy copy)
{
    if constexpr (USE == GRAD) {
        const int64_t over = static_cast<int64_t>(blockIdx.x) - tiles_m * tiles_n;
        if (over >= 0) {
            copy_rows<typename T::M>(copy, over * T::NT + threadIdx.x, (gridDim.x - tiles_m * tiles_n) * T::NT);
            return;
        }
    }
    int64_t tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, group, tm, tn);
    const int64_t k0 = blockIdx.y * k_split;
    const int64_t m0 = m_first + tm * T::BM, n0 = n_first + tn * T::BN;
    T tile;
    acc4 acc[T::TM][T::TN];
    const int64_t k = K - k0 < k_split ? K - k0 : k_split;
    tile.run(acc, a, b, parts, m0, n0, k0, k);
    // An operand without finite parts (forward 512 x 21841 x 4096: the check costs
    // nothing measurable, one class of -inf 0.62 -> 0.80 ms, one in every tile 1.24).
    if constexpr (T::SPLIT) {
        const int rows = static_cast<int>(M - m0 < T::BM ? M - m0 : T::BM);
        const int cols = static_cast<int>(N - n0 < T::BN ? N - n0 : T::BN);
        if (__builtin_amdgcn_readfirstlane(__syncthreads_or(any_not_finite<T>(acc, rows, cols)))) {
            typename T::InFp32 again;
            again.run(acc, a, b, parts, m0, n0, k0, k);
        }
    }
    finish<T, USE>(acc, o, m0, n0, tn, M, N, static_cast<int>(blockIdx.y));
}

// ---------------------------------------------------------------------------
// Joining and preparing.
// ---------------------------------------------------------------------------
constexpr int THREADS = 256;

__device__ __forceinline__ Run wave_join(Run r)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1)
        r = join(r, Run{__shfl_xor(r.m, m), __shfl_xor(r.s, m)});
    return r;
}

// One wave a row: lse and loss from the tiles' partial runs (main_count of them
// for the first main_rows rows, rest_count for the others), each lane taking
// every 64th, then joined across the wave in a fixed order.
__global__ __launch_bounds__(THREADS) void loss_kernel(const Run* __restrict__ part, int64_t nparts,
                                                       int64_t main_rows, int64_t main_count, int64_t rest_count,
                                                       const float* __restrict__ target_logit,
                                                       const int64_t* __restrict__ target, int64_t T, int64_t V,
                                                       float* __restrict__ loss, float* __restrict__ lse_out)
{
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (THREADS / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= T)
        return;
    Run r{-INFINITY, 0.f};
    const int64_t count = row < main_rows ? main_count : rest_count;
    for (int64_t p = lane; p < count; p += 64)
        r = join(r, part[row * nparts + p]);
    r = wave_join(r);
    if (lane == 0) {
        const float lse = lse_of(r);
        lse_out[row] = lse;
        loss[row] = counts(target[row], V) ? lse - target_logit[row] : 0.f;
    }
}

// The factor form, and the forward pass where the rows are few: the logits are
// the sums of the product's splits of k, and pass through memory (in the factor
// form G replaces them in U).  Rows of up to ROW_MOST values are a workgroup's:
// a thread holds EACH groups of four neighbours, and all loads of a split are
// in flight together.  Longer rows go in chunks, so that a few of them fill the
// GPU too: one kernel leaves every chunk's run, another joins a row's runs and
// turns each chunk into G.
constexpr int64_t ROW_MOST = 16384;
constexpr int CHUNK_EACH = 4, CHUNK = THREADS * 4 * CHUNK_EACH;

// n values at p, past them `past`.
__device__ __forceinline__ acc4 get4(const float* p, int n, float past)
{
    acc4 v = {past, past, past, past};
    if (n >= 4) {
        v = *reinterpret_cast<const f4a*>(p);
    } else if (n > 0) {
        v[0] = p[0];
        if (n > 1)
            v[1] = p[1];
        if (n > 2)
            v[2] = p[2];
    }
    return v;
}

// EACH groups of a row's (or chunk's) n logits from s on, the splits' sums, past
// n -inf; and the run of what the thread holds.
template <int NT, int EACH>
__device__ __forceinline__ Run held_logits(const float* s, int n, int splits, int64_t stride, acc4 (&held)[EACH])
{
    const int at = 4 * static_cast<int>(threadIdx.x);
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        held[e] = get4(s + at + 4 * NT * e, n - at - 4 * NT * e, -INFINITY);
    for (int z = 1; z < splits; ++z) {
        acc4 x[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            x[e] = get4(s + z * stride + at + 4 * NT * e, n - at - 4 * NT * e, 0.f);
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            held[e] += x[e];
    }
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            top = fmaxf(top, held[e][i]);
    const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sum += exp_diff(held[e][i], from);   // past n: 0
    return Run{top, sum};
}

template <int NT>
__device__ __forceinline__ Run group_join(Run r)
{
    __shared__ Run runs[NT / 64];
    r = wave_join(r);
    __syncthreads();   // the row before has read its runs
    if ((threadIdx.x & 63) == 0)
        runs[threadIdx.x >> 6] = r;
    __syncthreads();
    return wave_join((threadIdx.x & 63) < NT / 64 ? runs[threadIdx.x & 63] : Run{-INFINITY, 0.f});
}

// What turns a row's logits into G (as finish_grad does).
struct RowGrad {
    bool has;
    float lse, dloss;
};

// Four of a row's values from column v on: G to U and to the operand of dX (fp32,
// or bf16 in two parts `plane` apart; `g` up to ldg values, zeros past V).
template <typename G>
__device__ __forceinline__ void put_grad(const RowGrad& q, acc4 x, int v, int V, int ldg, int64_t plane,
                                         int64_t target, float* U, G* g)
{
    const int64_t hit = q.has ? target - v : -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = q.has && v + i < V ? exp_diff(x[i], q.lse) * q.dloss : 0.f;
        if (hit == i)
            x[i] -= q.dloss;
    }
    if (v < V)
        put4(U + v, x, V - v);
    if (v < ldg) {   // ldg: a multiple of eight
        if constexpr (sizeof(G) == 2) {
            const b4 h = __builtin_convertvector(x, b4);
            *reinterpret_cast<b4*>(g + v) = h;
            *reinterpret_cast<b4*>(g + plane + v) = __builtin_convertvector(x - __builtin_convertvector(h, acc4), b4);
        } else
            *reinterpret_cast<acc4*>(g + v) = x;
    }
}

template <typename G, int NT, int EACH, bool FACTOR>
__global__ __launch_bounds__(NT) void row_kernel(const float* logits, int splits, int64_t T, int64_t stride,
                                                 const int64_t* __restrict__ target, const float* __restrict__ dloss,
                                                 int V, float* __restrict__ loss, float* __restrict__ lse_out,
                                                 float* U, G* __restrict__ g, int ldg, int64_t plane)
{
    const int at = 4 * static_cast<int>(threadIdx.x);
    for (int64_t row = blockIdx.x; row < T; row += gridDim.x) {
        acc4 held[EACH];
        const int64_t t = target[row];
        const bool has = counts(t, V);
        const float d = FACTOR && has ? dloss[row] : 0.f;
        const float lse = lse_of(group_join<NT>(held_logits<NT, EACH>(logits + row * V, V, splits, stride, held)));
        if (threadIdx.x == 0) {
            if (!FACTOR)
                lse_out[row] = lse;
            if (!has)
                loss[row] = 0.f;
        }
        const RowGrad q{has, lse, d};
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int v = at + 4 * NT * e;
            if (has && t >= v && t < v + 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t == v + i)
                        loss[row] = lse - held[e][i];
            }
            if constexpr (FACTOR)
                put_grad(q, held[e], v, V, ldg, plane, t, U + row * V, g + row * ldg);
        }
    }
}

// A chunk's run; in the factor form of several splits also their sums, to U.
template <bool FACTOR>
__global__ __launch_bounds__(THREADS) void chunk_kernel(const float* logits, int splits, int64_t T, int64_t stride,
                                                        int chunks, const int64_t* __restrict__ target, int V,
                                                        Run* __restrict__ part, float* __restrict__ target_logit,
                                                        float* U)
{
    const int at = 4 * static_cast<int>(threadIdx.x);
    for (int64_t b = blockIdx.x; b < T * chunks; b += gridDim.x) {
        const int64_t row = b / chunks, from = (b - row * chunks) * CHUNK;
        const int n = static_cast<int>(V - from < CHUNK ? V - from : CHUNK);
        acc4 held[CHUNK_EACH];
        const Run r = group_join<THREADS>(
            held_logits<THREADS, CHUNK_EACH>(logits + row * V + from, n, splits, stride, held));
        if (threadIdx.x == 0)
            part[b] = r;
        const int64_t t = target[row] - from;
#pragma unroll
        for (int e = 0; e < CHUNK_EACH; ++e) {
            const int v = at + 4 * THREADS * e;
            if (t >= v && t < v + 4 && t < n) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t == v + i)
                        target_logit[row] = held[e][i];
            }
            if (FACTOR && splits > 1 && v < n)
                put4(U + row * V + from + v, held[e], n - v);
        }
    }
}

template <typename G>
__global__ __launch_bounds__(THREADS) void chunk_grad_kernel(const Run* __restrict__ part, int64_t T, int chunks,
                                                             const float* __restrict__ target_logit,
                                                             const int64_t* __restrict__ target,
                                                             const float* __restrict__ dloss, int V,
                                                             float* __restrict__ loss, float* __restrict__ U,
                                                             G* __restrict__ g, int ldg, int64_t plane)
{
    const int at = 4 * static_cast<int>(threadIdx.x);
    for (int64_t b = blockIdx.x; b < T * chunks; b += gridDim.x) {
        const int64_t row = b / chunks;
        const int from = static_cast<int>(b - row * chunks) * CHUNK;
        acc4 x[CHUNK_EACH];
#pragma unroll
        for (int e = 0; e < CHUNK_EACH; ++e)
            x[e] = get4(U + row * V + from + at + 4 * THREADS * e, V - from - at - 4 * THREADS * e, 0.f);
        Run r{-INFINITY, 0.f};
        for (int p = threadIdx.x & 63; p < chunks; p += 64)
            r = join(r, part[row * chunks + p]);
        const float lse = lse_of(wave_join(r));
        const int64_t t = target[row];
        const bool has = counts(t, V);
        if (from == 0 && threadIdx.x == 0)
            loss[row] = has ? lse - target_logit[row] : 0.f;
        const RowGrad q{has, lse, has ? dloss[row] : 0.f};
        // The last chunk also clears what is between V and the operand's row end.
#pragma unroll
        for (int e = 0; e < CHUNK_EACH; ++e)
            put_grad(q, x[e], from + at + 4 * THREADS * e, V, ldg, plane, t, U + row * V, g + row * ldg);
    }
}

template <typename E>
__global__ __launch_bounds__(THREADS) void lay_out_kernel(RowCopy c)
{
    copy_rows<E>(c, static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x,
                 static_cast<int64_t>(gridDim.x) * THREADS);
}

// The splits' sums in order, rounded once to the result's type.  A result of
// few values is bound by the splits' latency: eight splits are loaded together.
template <typename O>
__global__ __launch_bounds__(THREADS) void join_splits_kernel(const float* __restrict__ part, int splits,
                                                              int64_t stride, int64_t n, O* __restrict__ out)
{
    constexpr int AT_ONCE = 8;
    const int64_t groups = (n + 3) / 4, step = static_cast<int64_t>(gridDim.x) * THREADS;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; q < groups; q += step) {
        const int64_t at = 4 * q;
        const int left = static_cast<int>(n - at < 4 ? n - at : 4);
        acc4 v = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; s += AT_ONCE) {
            acc4 x[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                x[k] = s + k < splits ? get4(part + (s + k) * stride + at, left, 0.f) : acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                v += x[k];
        }
        if constexpr (sizeof(O) == 2)
            put4(out + at, __builtin_convertvector(v, b4), left);
        else
            put4(out + at, v, left);
    }
}

// ---------------------------------------------------------------------------
// Host: tile shapes, splits, workspaces.
// ---------------------------------------------------------------------------
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
unsigned grid_for(int64_t work) { return static_cast<unsigned>(std::min<int64_t>(work, 1 << 20)); }

constexpr int64_t ALIGN = 256;   // bytes between workspace arrays

struct Arena {
    char* base;
    int64_t at = 0;
    void* take(int64_t bytes)
    {
        void* p = base ? base + at : nullptr;
        at += round_up(std::max<int64_t>(bytes, 1), ALIGN);
        return p;
    }
};

// Tile shapes: rows x columns of a workgroup, of a wave, stages.  All take 128
// bytes of k a step.  THIN is for 32 rows or fewer; of the others the larger
// read less per product and the smaller fill the GPU with fewer tiles.  fp32 is
// multiplied by the fp32 matrix instructions up to 64 x 128, in bf16 parts at
// 128 x 128 (8192 x 8192 x 4096: 134 against 206 TFLOP/s; on 64 x 64 tiles a
// step waits for its parts, 127 against 114).
enum ShapeKind { THIN, SMALL, HALF, SQUARE, TALL, LARGE };

template <typename E, bool AK, bool BK>
using Thin = Tile<E, AK, BK, 32, 64, 32, 16, 4>;
template <typename E, bool AK, bool BK>
using Small = Tile<E, AK, BK, 64, 64, 32, 32, 3>;
template <typename E, bool AK, bool BK>
using Half = Tile<E, AK, BK, 64, 128, 64, 32, 3>;
template <typename E, bool AK, bool BK>
using Square = Tile<E, AK, BK, 128, 128, 64, 64, 2>;
template <typename E, bool AK, bool BK>
using Tall = Tile<E, AK, BK, 256, 192, 128, 48, 2>;
template <typename E, bool AK, bool BK, bool SPREAD = false>
using Large = Tile<E, AK, BK, 256, 256, 128, 64, 2, SPREAD>;

// What a shape costs, as measured (products over K = 4096, 512 and 64 on 256, 512
// and 768 tiles): microseconds of a step with one, two, three workgroups on a
// CU, bf16 and fp32, and of a tile's start; a CU writes 24 KB of results per
// microsecond.
struct Shape {
    int bm, bn, waves_n, per_cu;
    double step_us[2][3], tile_us;
};
constexpr Shape SHAPES[] = {
    {32, 64, 4, 3, {{0.29, 0.46, 0.66}, {0.50, 0.74, 1.02}}, 3.5},
    {64, 64, 2, 3, {{0.30, 0.42, 0.58}, {0.65, 1.09, 1.56}}, 4.0},
    {64, 128, 4, 2, {{0.42, 0.63, 0.}, {1.12, 2.03, 0.}}, 4.5},
    {128, 128, 2, 2, {{0.78, 1.00, 0.}, {1.66, 2.78, 0.}}, 5.0},
    {256, 192, 4, 1, {{1.25, 0., 0.}, {0., 0., 0.}}, 6.0},
    {256, 256, 4, 1, {{1.57, 0., 0.}, {0., 0., 0.}}, 6.0},
};

// A value's end in a tile, in bytes written or the like: G in bf16 parts counts
// its arithmetic too.
template <typename E, Use USE>
constexpr double OUT_BYTES = USE == STATS ? 0.5 : USE == GRAD && sizeof(E) == 2 ? 8.0 : 4.0;

// How an M x N product is computed: the first `rows` x `cols` of it in tiles of
// `kind`; rows past them, or columns (never both), in tiles of `rest`; k split
// `splits` ways, whose sums a kernel of their own adds.
struct Choice {
    ShapeKind kind;
    int64_t splits;
    double us;
    int64_t rows, cols;
    ShapeKind rest;
};

// Whole rounds of workgroups over the GPU and a last one that is not full.
inline double tiles_us(const Shape& s, int type, int64_t M, int64_t N, double steps, int z, double out_bytes)
{
    const int cus = device_cu_count();
    const int64_t tiles = ceil_div(M, s.bm) * ceil_div(N, s.bn) * z;
    const int64_t full = tiles / (s.per_cu * cus);
    const int over = static_cast<int>(tiles - full * (s.per_cu * cus));
    const double out = out_bytes * s.bm * s.bn / 24e3;
    double us = static_cast<double>(full) * (steps * s.step_us[type][s.per_cu - 1] + s.tile_us + s.per_cu * out);
    if (over > 0) {
        const int n = (over - 1) / cus;
        us += steps * s.step_us[type][n] + s.tile_us + (n + 1) * out;
    }
    return us;
}

// The smaller shape that finishes first (its estimate in `us`).
inline ShapeKind rest_shape(int type, int64_t M, int64_t N, double steps, int z, double out_bytes, double& us)
{
    ShapeKind by = SMALL;
    us = 1e30;
    for (int k = M <= 32 ? THIN : SMALL; k <= LARGE; ++k) {
        if (SHAPES[k].step_us[type][0] == 0.0)
            continue;
        const double x = tiles_us(SHAPES[k], type, M, N, steps, z, out_bytes);
        if (x < us) {
            us = x;
            by = static_cast<ShapeKind>(k);
        }
    }
    return by;
}

// The choice that finishes M x N values over K of k first, by these estimates;
// never less than reading both operands takes.
template <typename E, Use USE>
Choice choose(int64_t M, int64_t N, int64_t K, int count, bool may_split)
{
    constexpr int TYPE = sizeof(E) / 4;
    constexpr double OUT = OUT_BYTES<E, USE>;
    if (M == 0 || N == 0)   // nothing is launched
        return Choice{SMALL, 1, 0.0, M, N, SMALL};
    const int64_t steps = ceil_div(std::max<int64_t>(K, 1), 128 / static_cast<int64_t>(sizeof(E)));
    const int64_t cus = device_cu_count();
    const double reading = static_cast<double>((M + N) * K) * sizeof(E) / 4.8e6;
    const double sums = 4.0 * static_cast<double>(M * N) / 4e6;   // written or read once, at 4 TB/s
    Choice best{SMALL, 1, 1e30, M, N, SMALL};
    for (int k = M <= 32 ? THIN : SMALL; k <= LARGE; ++k) {
        const Shape& s = SHAPES[k];
        if (s.step_us[TYPE][0] == 0.0)
            continue;
        const int64_t slots = s.per_cu * cus, down = ceil_div(M, s.bm), across = ceil_div(N, s.bn);
        const int most = may_split ? static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(32, steps / 4))) : 1;
        const int64_t over = M % s.bm;
        // All of it in this shape; or (large shapes) without a ragged rest of
        // rows, at most half a tile's; or without the columns past the last full
        // round of workgroups.  k whole, or split into what comes to whole rounds.
        for (int form = 0; form < (k >= SQUARE ? 3 : 1); ++form) {
            if (form == 1 && (over == 0 || over > s.bm / 2 || M < s.bm))
                continue;
            const int64_t rows = form == 1 ? M - over : M;
            const int64_t tiles = form == 1 ? (down - 1) * across : down * across;
            for (int round = 0; round <= 4; ++round) {
                const int z = round == 0 ? 1 : static_cast<int>(std::min<int64_t>(most, round * slots / tiles));
                if (z < 1 || (round > 0 && z == 1))
                    continue;
                int64_t cols = N;
                if (form == 2) {
                    const int64_t full = tiles * z / slots * slots / z / down;   // columns of tiles in full rounds
                    if (full < 1 || full >= across)
                        continue;
                    cols = full * s.bn;
                }
                const double each = static_cast<double>((steps + z - 1) / z * count);
                // The splits' sums are written (once is counted), read and written, and take a launch.
                const double joined = z > 1 ? 5.0 + (z + 1) * sums : 0.0;
                double us = tiles_us(s, TYPE, rows, cols, each, z, OUT);
                ShapeKind by = SMALL;
                if (form > 0 && us + joined < best.us) {
                    // A launch of its own: 4 us, and its workgroups no longer
                    // start as the first ones of the last round end (a round's
                    // sixth: 512 x 21841 x 4096 fp32 531 us whole, 588 so).
                    double rest;
                    by = form == 1 ? rest_shape(TYPE, over, N, each, z, OUT, rest)
                                   : rest_shape(TYPE, M, N - cols, each, z, OUT, rest);
                    us += 4.0 + rest;
                    if (form == 2)
                        us += each * s.step_us[TYPE][s.per_cu - 1] / 6;
                }
                us = std::max(us, reading) + joined;
                if (us < best.us)
                    best = Choice{static_cast<ShapeKind>(k), z, us, rows, cols, by};
            }
        }
    }
    return best;
}

template <typename T, Use USE>
hipError_t launch_product(const Operand& a, const Operand& b, const Parts& p, const Out& o, int64_t m_first,
                          int64_t n_first, int64_t M, int64_t N, int64_t K, int64_t splits, hipStream_t s,
                          const RowCopy& copy)
{
    const int64_t tm = ceil_div(M - m_first, T::BM), tn = ceil_div(N - n_first, T::BN);
    const int64_t k_split = round_up(ceil_div(std::max<int64_t>(K, 1), splits), T::STEP);
    const int64_t copies = USE == GRAD && copy.out
                               ? std::min<int64_t>(ceil_div(copy.rows * (copy.ldo / GROUP), T::NT), 2 * device_cu_count())
                               : 0;
    product_kernel<T, USE><<<dim3(static_cast<unsigned>(tm * tn + copies), static_cast<unsigned>(splits)), T::NT, 0,
                             s>>>(a, b, p, o, m_first, n_first, M, N, K, k_split, tm, tn, 1024 / T::BM, copy);
    return hipGetLastError();
}

template <typename E, bool AK, bool BK, Use USE>
hipError_t product_part(ShapeKind kind, const Operand& a, const Operand& b, const Parts& p, const Out& o,
                        int64_t m_first, int64_t n_first, int64_t M, int64_t N, int64_t K, int64_t splits,
                        hipStream_t s, const RowCopy& copy)
{
    auto go = [&](auto* launch) { return launch(a, b, p, o, m_first, n_first, M, N, K, splits, s, copy); };
    switch (kind) {
    case THIN:
        return go(launch_product<Thin<E, AK, BK>, USE>);
    case SMALL:
        return go(launch_product<Small<E, AK, BK>, USE>);
    case HALF:
        return go(launch_product<Half<E, AK, BK>, USE>);
    case SQUARE:
        // (The choice of shapes, and with it the workspace, is the split's in
        // either arithmetic: the setting may change between query and call.)
        if constexpr (sizeof(E) == 4)
            if (sf_arithmetic() != POSEIDON_SF_FP32)
                return go(launch_product<Square<Split32, AK, BK>, USE>);
        return go(launch_product<Square<E, AK, BK>, USE>);
    case TALL:
        if constexpr (sizeof(E) == 2)
            return go(launch_product<Tall<E, AK, BK>, USE>);
        break;
    case LARGE:
        if constexpr (sizeof(E) == 2)
            return go(launch_product<Large<E, AK, BK, USE == GRAD>, USE>);
        break;
    }
    return hipErrorInvalidValue;
}

// Runs that a row of N columns leaves, one a wave.
int64_t column_blocks(ShapeKind kind, int64_t N) { return ceil_div(N, SHAPES[kind].bn) * SHAPES[kind].waves_n; }

template <typename E, bool AK, bool BK, Use USE>
hipError_t product(const Choice& c, const Operand& a, const Operand& b, const Parts& p, const Out& o, int64_t M,
                   int64_t N, int64_t K, hipStream_t s, const RowCopy& copy = {})
{
    const hipError_t rc =
        product_part<E, AK, BK, USE>(c.kind, a, b, p, o, 0, 0, c.rows, c.cols, K, c.splits, s, copy);
    if (rc != hipSuccess || (c.rows == M && c.cols == N))
        return rc;
    if (c.rows < M)
        return product_part<E, AK, BK, USE>(c.rest, a, b, p, o, c.rows, 0, M, N, K, c.splits, s, RowCopy{});
    Out right = o;
    right.block_first = column_blocks(c.kind, c.cols);
    return product_part<E, AK, BK, USE>(c.rest, a, b, p, right, 0, c.cols, M, N, K, c.splits, s, RowCopy{});
}

// Products of parts, four bits each (A's, then B's): one; two, three of A with
// one of B.
constexpr Parts ONE{1, 0}, TWO_A{2, 0x10}, THREE_A{3, 0x210};

template <typename O>
hipError_t join_splits(const float* part, int64_t splits, int64_t n, O* out, hipStream_t s)
{
    join_splits_kernel<O><<<grid_for(ceil_div(n, THREADS * 4)), THREADS, 0, s>>>(part, static_cast<int>(splits), n,
                                                                                     n, out);
    return hipGetLastError();
}

// X or W as the caller has it is an operand where its rows lie on 4-byte
// boundaries (fp32 always); else it is laid out again.
template <typename I>
bool needs_copy(const void* p, int64_t D)
{
    return reinterpret_cast<uintptr_t>(p) % 4 != 0 || D * static_cast<int64_t>(sizeof(I)) % 4 != 0;
}

template <typename E>
hipError_t lay_out(const RowCopy& c, hipStream_t s)
{
    if (c.rows > 0)
        lay_out_kernel<E><<<grid_for(ceil_div(c.rows * (c.ldo / GROUP), THREADS)), THREADS, 0, s>>>(c);
    return hipGetLastError();
}

// So many rows are few: the logits of all classes are then small beside W, and
// the forward pass too takes them through memory, which lets k be split so that
// the GPU is full.
constexpr int64_t FEW_ROWS = 32;
constexpr int64_t PIECE_BYTES = int64_t(512) << 20;   // of G at a time

// How the three products of one piece are computed.
struct Pieces {
    Choice logits{}, dx{}, dw{};
    double us() const { return logits.us + dx.us + dw.us; }
};

struct Plan {
    bool by_row = false, own_x = false, own_w = false;
    int64_t ldd = 0;   // row length of what is laid out
    void* x = nullptr;
    void* clean_x = nullptr;   // backward: X without the rows that have no target
    void* w = nullptr;
    Choice logits{};      // forward and factor form
    Pieces full, last;    // backward: of the full pieces and the last one
    float* row_logits = nullptr;   // by row: splits x T x V
    Run* part = nullptr;           // else: a run per row and column block
    int64_t nparts = 0, main_runs = 0, rest_runs = 0;   // of a row; of the main rows; of the others
    float* target_logit = nullptr;
    void* g = nullptr;
    int64_t piece = 0, ldg = 0;
    float* dx = nullptr;
    float* dw = nullptr;
    int64_t bytes = 0;
};

// dW = G^T X: G is fp32, or (bf16 X) its three exact bf16 parts.
template <typename E>
constexpr Parts DW_PARTS = sizeof(E) == 2 ? THREE_A : ONE;
// dX = G W: of a bf16 G the first two parts, which leave out 2^-16 of each entry.
// One part (2^-8, the target's entry exact) hides below dX's own rounding where
// W's rows average to 0, but a row of G sums to 0, so what W's rows share cancels
// in exact arithmetic and what rounding left of it does not: with a shared
// component of 30 times their spread dX was off by 3.6 to 5.8 times its rounding.
// The second part costs a product (backward 4097 x 50001 x 1024 2.20 -> 2.57 ms,
// factors 32 x 21841 x 4096 95 -> 101 us).
template <typename E>
constexpr Parts DX_PARTS = sizeof(E) == 2 ? TWO_A : ONE;

template <typename E>
Pieces pieces(int64_t T, int64_t rows, int64_t D)
{
    return Pieces{choose<E, GRAD>(T, rows, D, 1, false), choose<E, STORE>(T, D, rows, DX_PARTS<E>.count, true),
                  choose<E, STORE>(rows, D, T, DW_PARTS<E>.count, true)};
}

template <typename E>
Plan make_plan(int op, const void* X, const void* W, int64_t T, int64_t V, int64_t D, char* base)
{
    constexpr int64_t SZ = sizeof(E);
    Plan p;
    Arena a{base};
    p.ldd = round_up(D, GROUP);
    p.own_x = needs_copy<E>(X, D);
    p.own_w = needs_copy<E>(W, D);
    if (p.own_x)
        p.x = a.take(T * p.ldd * SZ);
    if (op == POSEIDON_XENT_BACKWARD)
        p.clean_x = a.take(T * p.ldd * SZ);
    if (p.own_w)
        p.w = a.take(V * p.ldd * SZ);
    p.by_row = op == POSEIDON_XENT_FACTOR || (op == POSEIDON_XENT_FORWARD && T <= FEW_ROWS);
    p.logits = p.by_row ? choose<E, STORE>(T, V, D, 1, true) : choose<E, STATS>(T, V, D, 1, false);
    if (p.by_row) {
        if (op == POSEIDON_XENT_FORWARD || p.logits.splits > 1)
            p.row_logits = static_cast<float*>(a.take(p.logits.splits * T * V * 4));
        if (V > ROW_MOST) {
            p.part = static_cast<Run*>(a.take(T * ceil_div(V + GROUP, CHUNK) * static_cast<int64_t>(sizeof(Run))));
            p.target_logit = static_cast<float*>(a.take(T * 4));
        }
    } else if (op != POSEIDON_XENT_BACKWARD) {
        p.main_runs = column_blocks(p.logits.kind, p.logits.cols);
        if (p.logits.cols < V)
            p.main_runs += column_blocks(p.logits.rest, V - p.logits.cols);
        p.rest_runs = p.logits.rows < T ? column_blocks(p.logits.rest, V) : 0;
        p.nparts = std::max(p.main_runs, p.rest_runs);
        p.part = static_cast<Run*>(a.take(T * p.nparts * static_cast<int64_t>(sizeof(Run))));
        p.target_logit = static_cast<float*>(a.take(T * 4));
    }
    if (op == POSEIDON_XENT_FORWARD) {
        p.bytes = a.at;
        return p;
    }
    // G: fp32, or in bf16 parts (for a factor's bf16 dX two of them).
    const int64_t g_value = SZ == 4 || op == POSEIDON_XENT_FACTOR ? 4 : 6;
    p.piece = round_up(V, GROUP);
    p.full.dx = choose<E, STORE>(T, D, V, DX_PARTS<E>.count, true);
    if (op == POSEIDON_XENT_BACKWARD) {
        // Pieces of the vocabulary within the budget: equal ones, or as many
        // classes as make whole rounds of dW's largest tiles and a rest;
        // whichever the choices' estimates make cheapest.
        const int64_t most = std::max<int64_t>(PIECE_BYTES / g_value / std::max<int64_t>(T, 1) / 256, 1) * 256;
        const int64_t fewest = ceil_div(V, most), across = ceil_div(D, 256);
        const int64_t rounds = most / 256 * across / device_cu_count();
        double best = 1e30;
        for (int i = 0; i < (fewest > 1 ? 6 : 1); ++i) {
            const int64_t even = round_up(ceil_div(V, fewest + i), 256);
            const int64_t piece = fewest == 1 ? round_up(V, GROUP)
                                  : i < 4     ? even
                                              : (rounds - (i - 4)) * device_cu_count() / across * 256;
            if (piece < 256 && fewest > 1)
                continue;
            const int64_t rows = std::min(piece, V), over = V % rows;
            const Pieces full = pieces<E>(T, rows, D), last = over ? pieces<E>(T, over, D) : Pieces{};
            const double us = static_cast<double>(V / rows) * full.us() + last.us();
            if (us < best) {
                best = us;
                p.piece = piece;
                p.full = full;
                p.last = over ? last : full;
            }
        }
        // The rest adds to the full pieces' sums: to no more of them than there are.
        p.last.dx.splits = std::min(p.last.dx.splits, p.full.dx.splits);
        const int64_t rows = std::min(p.piece, V);
        const int64_t dw_sums = std::max(p.full.dw.splits > 1 ? p.full.dw.splits * rows : 0,
                                         p.last.dw.splits > 1 ? p.last.dw.splits * (V % rows) : 0);
        if (dw_sums > 0)
            p.dw = static_cast<float*>(a.take(dw_sums * D * 4));
    }
    // Rows of a multiple of 4 KB would put the 16 rows of a store on one memory
    // channel (G of 4096 x 16384, in parts: 222 us, with 512 bytes more 200).
    p.ldg = p.piece + (p.piece * (SZ == 4 ? 4 : 2) % 4096 == 0 ? 512 / SZ : 0);
    p.g = a.take(T * p.ldg * g_value);
    if (p.full.dx.splits > 1 || (p.piece < V && SZ == 2))
        p.dx = static_cast<float*>(a.take(p.full.dx.splits * T * D * 4));
    p.bytes = a.at;
    return p;
}

#define POSEIDON_TRY(x)              \
    do {                             \
        const hipError_t rc_ = (x);  \
        if (rc_ != hipSuccess)       \
            return rc_;              \
    } while (0)

// X and W as operands, laid out where their rows' places ask for it.
template <typename E>
hipError_t operands(const Plan& p, const E* X, const E* W, int64_t T, int64_t V, int64_t D, Operand& x, Operand& w,
                    hipStream_t s)
{
    if (p.own_x)
        POSEIDON_TRY(lay_out<E>(RowCopy{X, T, D, p.ldd, nullptr, V, p.x}, s));
    if (p.own_w)
        POSEIDON_TRY(lay_out<E>(RowCopy{W, V, D, p.ldd, nullptr, V, p.w}, s));
    x = Operand{p.own_x ? p.x : X, p.own_x ? p.ldd : D, T, 0};
    w = Operand{p.own_w ? p.w : W, p.own_w ? p.ldd : D, V, 0};
    return hipSuccess;
}

// G's rows end on whole chunks (zeros past V).
template <typename E>
int64_t whole_chunks(int64_t k)
{
    return round_up(k, 16 / static_cast<int64_t>(sizeof(E)));
}

template <typename E>
hipError_t row_logits(const Plan& p, const Operand& x, const Operand& w, int64_t T, int64_t V, int64_t D, float* U,
                      hipStream_t s)
{
    Out o{};
    o.c = p.row_logits ? p.row_logits : U;
    o.ldc = V;
    o.split_stride = T * V;
    return product<E, true, true, STORE>(p.logits, x, w, ONE, o, T, V, D, s);
}

hipError_t join_runs(const Plan& p, int64_t stride, int64_t main_rows, int64_t main_count, int64_t rest_count,
                     const int64_t* target, int64_t T, int64_t V, float* loss, float* lse, hipStream_t s)
{
    loss_kernel<<<static_cast<unsigned>(ceil_div(T, THREADS / 64)), THREADS, 0, s>>>(
        p.part, stride, main_rows, main_count, rest_count, p.target_logit, target, T, V, loss, lse);
    return hipGetLastError();
}

// Losses (and lse, or G) from the logits in memory.
template <typename G, bool FACTOR>
hipError_t rows_done(const Plan& p, const int64_t* target, const float* dloss, int64_t T, int64_t V, float* loss,
                     float* lse, float* U, hipStream_t s)
{
    const float* logits = p.row_logits ? p.row_logits : U;
    const int splits = static_cast<int>(p.logits.splits), v = static_cast<int>(V), ldg = static_cast<int>(p.ldg);
    G* g = static_cast<G*>(p.g);
    if (V <= ROW_MOST) {
        auto run = [&](auto* k, int threads) {
            k<<<grid_for(T), threads, 0, s>>>(logits, splits, T, T * V, target, dloss, v, loss, lse, U, g, ldg,
                                              T * p.ldg);
        };
        // Groups of eight end the operand's rows, so a row's last group counts whole.
        const int64_t values = round_up(V, GROUP);
        if (values <= 1024)
            run(row_kernel<G, 256, 1, FACTOR>, 256);
        else if (values <= 4096)
            run(row_kernel<G, 256, 4, FACTOR>, 256);
        else
            run(row_kernel<G, 1024, 4, FACTOR>, 1024);
        return hipGetLastError();
    }
    const int chunks = static_cast<int>(ceil_div(round_up(V, GROUP), CHUNK));
    chunk_kernel<FACTOR><<<grid_for(T * chunks), THREADS, 0, s>>>(logits, splits, T, T * V, chunks, target, v, p.part,
                                                                  p.target_logit, U);
    POSEIDON_TRY(hipGetLastError());
    if constexpr (FACTOR) {
        chunk_grad_kernel<G><<<grid_for(T * chunks), THREADS, 0, s>>>(p.part, T, chunks, p.target_logit, target, dloss,
                                                                     v, loss, U, g, ldg, T * p.ldg);
        return hipGetLastError();
    } else {
        return join_runs(p, chunks, T, chunks, chunks, target, T, V, loss, lse, s);
    }
}

// Losses and lse without keeping logits.
template <typename E>
hipError_t losses(const Plan& p, const Operand& x, const Operand& w, const int64_t* target, int64_t T, int64_t V,
                  int64_t D, float* loss, float* lse, hipStream_t s)
{
    Out o{};
    o.part = p.part;
    o.nparts = p.nparts;
    o.target_logit = p.target_logit;
    o.target = target;
    POSEIDON_TRY((product<E, true, true, STATS>(p.logits, x, w, ONE, o, T, V, D, s)));
    return join_runs(p, p.nparts, p.logits.rows, p.main_runs, p.rest_runs, target, T, V, loss, lse, s);
}

template <typename E>
hipError_t forward_typed(const E* X, const E* W, const int64_t* target, int64_t T, int64_t V, int64_t D, float* loss,
                         float* lse, char* ws, hipStream_t s)
{
    const Plan p = make_plan<E>(POSEIDON_XENT_FORWARD, X, W, T, V, D, ws);
    Operand x, w;
    POSEIDON_TRY(operands(p, X, W, T, V, D, x, w, s));
    if (!p.by_row)
        return losses<E>(p, x, w, target, T, V, D, loss, lse, s);
    POSEIDON_TRY(row_logits<E>(p, x, w, T, V, D, nullptr, s));
    return rows_done<E, false>(p, target, nullptr, T, V, loss, lse, nullptr, s);
}

// dX = G W for one piece of the vocabulary (the first replaces, the others add).
template <typename E>
hipError_t input_gradient(const Plan& p, const Operand& g, const Operand& w, int64_t T, int64_t V, int64_t D,
                          int64_t v0, int64_t vp, E* dX, hipStream_t s)
{
    constexpr bool BF16 = sizeof(E) == 2;
    const bool first = v0 == 0, last = v0 + vp == V;
    const Choice& c = vp == std::min(p.piece, V) ? p.full.dx : p.last.dx;
    Out o{};
    o.c = p.dx ? static_cast<void*>(p.dx) : static_cast<void*>(dX);
    o.ldc = D;
    o.split_stride = T * D;
    o.bf16 = BF16 && !p.dx;
    o.add = !first;
    POSEIDON_TRY((product<E, true, false, STORE>(c, g, w, DX_PARTS<E>, o, T, D, whole_chunks<E>(vp), s)));
    return last && p.dx ? join_splits(p.dx, p.full.dx.splits, T * D, dX, s) : hipSuccess;
}

// G of the classes v0 .. v0 + vp.
template <typename E>
hipError_t logit_gradient(const Plan& p, const Operand& x, const Operand& w, const int64_t* target, const float* lse,
                          const float* dloss, int64_t T, int64_t V, int64_t D, int64_t v0, int64_t vp,
                          const RowCopy& copy, hipStream_t s)
{
    Out o{};
    o.target = target;
    o.lse = lse;
    o.dloss = dloss;
    o.g = p.g;
    o.ldg = p.ldg;
    o.g_plane = T * p.ldg;
    o.v0 = v0;
    o.V = V;
    const Choice& c = vp == std::min(p.piece, V) ? p.full.logits : p.last.logits;
    return product<E, true, true, GRAD>(c, x, w, ONE, o, T, vp, D, s, copy);
}

template <typename E>
hipError_t backward_typed(const E* X, const E* W, const int64_t* target, const float* lse, const float* dloss,
                          int64_t T, int64_t V, int64_t D, E* dX, float* dW, char* ws, hipStream_t s)
{
    const Plan p = make_plan<E>(POSEIDON_XENT_BACKWARD, X, W, T, V, D, ws);
    Operand x, w;
    POSEIDON_TRY(operands(p, X, W, T, V, D, x, w, s));
    const Operand g{p.g, p.ldg, T, T * p.ldg};
    // dW multiplies G's zero rows too: whatever X holds where a row has no
    // target must not reach it.
    const RowCopy clean{X, T, D, p.ldd, target, V, p.clean_x};
    const Operand cx{p.clean_x, p.ldd, T, 0};
    for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
        const int64_t vp = std::min(p.piece, V - v0);
        const Operand wp{static_cast<const E*>(w.p) + v0 * w.ld, w.ld, vp, 0};
        if (T > 0) {
            POSEIDON_TRY(logit_gradient<E>(p, x, wp, target, lse, dloss, T, V, D, v0, vp, v0 == 0 ? clean : RowCopy{}, s));
            POSEIDON_TRY((input_gradient<E>(p, g, wp, T, V, D, v0, vp, dX, s)));
        }
        const Choice& c = vp == std::min(p.piece, V) ? p.full.dw : p.last.dw;
        const bool sums = c.splits > 1;
        Out o{};
        o.c = sums ? p.dw : dW + v0 * D;
        o.ldc = D;
        o.split_stride = vp * D;
        POSEIDON_TRY((product<E, false, false, STORE>(c, g, cx, DW_PARTS<E>, o, vp, D, T, s)));
        if (sums)
            POSEIDON_TRY(join_splits(p.dw, c.splits, vp * D, dW + v0 * D, s));
    }
    return hipSuccess;
}

template <typename E>
hipError_t factor_typed(const E* X, const E* W, const int64_t* target, const float* dloss, int64_t T, int64_t V,
                        int64_t D, float* loss, float* U, E* dX, char* ws, hipStream_t s)
{
    const Plan p = make_plan<E>(POSEIDON_XENT_FACTOR, X, W, T, V, D, ws);
    Operand x, w;
    POSEIDON_TRY(operands(p, X, W, T, V, D, x, w, s));
    POSEIDON_TRY(row_logits<E>(p, x, w, T, V, D, U, s));
    POSEIDON_TRY((rows_done<E, true>(p, target, dloss, T, V, loss, nullptr, U, s)));
    return input_gradient<E>(p, Operand{p.g, p.ldg, T, T * p.ldg}, w, T, V, D, 0, V, dX, s);
}

}  // namespace

int64_t xent_workspace(int32_t op, const void* X, const void* W, int64_t T, int64_t V, int64_t D, int32_t dtype)
{
    return dtype == POSEIDON_BF16 ? make_plan<__bf16>(op, X, W, T, V, D, nullptr).bytes
                                  : make_plan<float>(op, X, W, T, V, D, nullptr).bytes;
}

hipError_t launch_xent_forward(const void* X, const void* W, const int64_t* target, int64_t T, int64_t V, int64_t D,
                               int32_t dtype, float* loss, float* lse, void* ws, hipStream_t stream)
{
    char* w = static_cast<char*>(ws);
    if (dtype == POSEIDON_BF16)
        return forward_typed(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W), target, T,
                                             V, D, loss, lse, w, stream);
    return forward_typed(static_cast<const float*>(X), static_cast<const float*>(W), target, T, V, D, loss, lse, w, stream);
}

hipError_t launch_xent_backward(const void* X, const void* W, const int64_t* target, const float* lse,
                                const float* dloss, int64_t T, int64_t V, int64_t D, int32_t dtype, void* dX,
                                float* dW, void* ws, hipStream_t stream)
{
    char* w = static_cast<char*>(ws);
    if (dtype == POSEIDON_BF16)
        return backward_typed(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W), target,
                                              lse, dloss, T, V, D, static_cast<__bf16*>(dX), dW, w, stream);
    return backward_typed(static_cast<const float*>(X), static_cast<const float*>(W), target, lse, dloss, T, V, D,
             static_cast<float*>(dX), dW, w, stream);
}

hipError_t launch_xent_factor(const void* X, const void* W, const int64_t* target, const float* dloss, int64_t T,
                              int64_t V, int64_t D, int32_t dtype, float* loss, float* U, void* dX, void* ws,
                              hipStream_t stream)
{
    char* w = static_cast<char*>(ws);
    if (dtype == POSEIDON_BF16)
        return factor_typed(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W), target,
                                            dloss, T, V, D, loss, U, static_cast<__bf16*>(dX), w, stream);
    return factor_typed(static_cast<const float*>(X), static_cast<const float*>(W), target, dloss, T, V, D, loss, U,
             static_cast<float*>(dX), w, stream);
}

}  // namespace poseidon
