// Softmax cross entropy fused with the classifier's product (include/poseidon.h
// gives the formulas): T rows X (T x D), V classes W (V x D),
//
//     s = X W^T,  lse_t = log sum_v exp s_tv,  loss_t = lse_t - s_t,target
//     G = (exp(s - lse) - onehot(target)) * dloss,  dX = G W,  dW = G^T X.
//
// The logits never leave the matrix cores' registers in the forward and the
// backward pass: the forward tile's epilogue reduces its columns to a running
// maximum and sum per row, and a second kernel joins them; the backward pass
// makes the logits again, a piece of the vocabulary at a time, turns them into
// G in the epilogue and multiplies the piece with W and X while it is in the
// last-level cache.  The factor form, for layers that are synchronised by
// sufficient factors, writes G whole, because there G is the payload.
//
// Bound: 2TVD operations a product on the matrix cores for many rows, reading
// W once for few.
#include <math.h>

#include "mfma_tile.h"

namespace poseidon {
namespace {

// e^x for x <= 0 or near it: 2^(x log2 e) with the product's rounding error put
// back, so that a small probability keeps fp32's relative accuracy.
__device__ __forceinline__ float exp_f(float x)
{
    const float y = x * 1.44269504f;
    const float r = fmaf(x, 1.44269504f, -y) + x * 1.92596299e-8f;   // the product's error, and log2(e)'s
    const float e = __builtin_amdgcn_exp2f(y);
    return y > -126.f && y < 128.f ? fmaf(e, r * 0.693147181f, e) : e;
}

// A running maximum and the sum of exponentials below it.
struct Run {
    float m, s;
};

__device__ __forceinline__ Run join(Run a, Run b)
{
    const float m = fmaxf(a.m, b.m);
    // A side without a finite maximum (no column, or all -inf) adds nothing.
    const float ea = a.m == -INFINITY ? 0.f : exp_f(a.m - m), eb = b.m == -INFINITY ? 0.f : exp_f(b.m - m);
    return Run{m, fmaf(a.s, ea, b.s * eb)};
}

__device__ __forceinline__ bool counts(int64_t target, int64_t V) { return target >= 0 && target < V; }

// ---------------------------------------------------------------------------
// What a tile does with its sums.  acc[i][j][r] of lane l is row
// m0 + 16 i + l % 16, column n0 + 16 j + 4 (l / 16) + r.
// ---------------------------------------------------------------------------
enum Use { STATS, LOGITS, GRAD, STORE };

struct Out {
    // STATS, LOGITS: per row and column block the running maximum and sum, and
    // the target's logit; LOGITS also the logits (`c`, ldc apart).
    Run* part;
    int64_t nparts;
    float* target_logit;
    const int64_t* target;
    // GRAD: the piece's G from lse and dloss, as bf16 parts (planes apart) or
    // fp32, columns v0 onwards of V.
    const float* lse;
    const float* dloss;
    void* g;
    int64_t ldg, g_plane;
    int32_t g_parts;      // bf16 parts written (1..3), or 0: fp32
    int64_t v0, V;
    // GRAD writes, and STORE of a bf16 dX reads, what rounding G to bf16 left of
    // each row's entry at its target: that entry is near -dloss where all others
    // are small, and its rounding error, the same in all of the row's dX, would
    // be most of the error.  STORE adds it times the target's row of W.
    float* target_rest;
    const void* W;
    int64_t ldw;
    // STORE: C (ldc apart), fp32 or bf16, added to what is there or not; with
    // several splits of k, split z's sums go to c + z * split_stride.
    void* c;
    int64_t ldc, split_stride;
    int32_t bf16, add;
};

// One row's four neighbours at p (any 4- or 2-byte boundary), n of them.
__device__ __forceinline__ void put4(float* p, acc4 v, int64_t n)
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

typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b4a __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ void put4(__bf16* p, b4 v, int64_t n)
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

template <typename T, Use USE>
__device__ __forceinline__ void finish(acc4 (&acc)[T::TM][T::TN], const Out& o, int64_t m0, int64_t n0, int64_t tile_n,
                                       int64_t M, int64_t N, int z)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int wm = (w / T::NWN) * T::WM, wn = (w % T::NWN) * T::WN;
    const int64_t n_lane = n0 + wn + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int64_t m = m0 + wm + 16 * i + (lane & 15);
        const bool row = m < M;
        if constexpr (USE == STATS || USE == LOGITS) {
            const int64_t t = row ? o.target[m] : -1;
            Run run{-INFINITY, 0.f};
#pragma unroll
            for (int j = 0; j < T::TN; ++j) {
                const int64_t n = n_lane + 16 * j;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = n + r < N ? acc[i][j][r] : -INFINITY;
                    run.m = fmaxf(run.m, x);
                }
            }
            // A NaN logit is not a maximum, but makes the sum one.
            run.m = fmaxf(run.m, __shfl_xor(run.m, 16));
            run.m = fmaxf(run.m, __shfl_xor(run.m, 32));
            const float from = run.m == -INFINITY ? 0.f : run.m;
#pragma unroll
            for (int j = 0; j < T::TN; ++j) {
                const int64_t n = n_lane + 16 * j;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n + r < N) {
                        run.s += exp_f(acc[i][j][r] - from);
                        if (n + r == t)
                            o.target_logit[m] = acc[i][j][r];
                    }
                if constexpr (USE == LOGITS)
                    if (row && n < N)
                        put4(static_cast<float*>(o.c) + m * o.ldc + n, acc[i][j], N - n);
            }
            run.s += __shfl_xor(run.s, 16);
            run.s += __shfl_xor(run.s, 32);
            if (row && lane < 16)
                o.part[m * o.nparts + tile_n * T::NWN + w % T::NWN] = run;
        } else if constexpr (USE == GRAD) {
            const int64_t t = row ? o.target[m] : -1;
            const bool has = row && counts(t, o.V);
            const float lse = row ? o.lse[m] : 0.f, d = row ? o.dloss[m] : 0.f;
#pragma unroll
            for (int j = 0; j < T::TN; ++j) {
                const int64_t n = n_lane + 16 * j;
                acc4 g;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = exp_f(acc[i][j][r] - lse) - (n + r + o.v0 == t ? 1.f : 0.f);
                    g[r] = has && n + r < N ? p * d : 0.f;   // past V: zeros up to the row's end
                }
                if (!row || n >= o.ldg)
                    continue;
                if (o.target_rest && has) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (n + r + o.v0 == t)
                            o.target_rest[m] = g[r] - static_cast<float>(static_cast<__bf16>(g[r]));
                }
                if (o.g_parts == 0) {
                    put4(static_cast<float*>(o.g) + m * o.ldg + n, g, 4);
                } else {
                    __bf16* at = static_cast<__bf16*>(o.g) + m * o.ldg + n;
                    for (int p = 0; p < o.g_parts; ++p) {
                        const b4 h = __builtin_convertvector(g, b4);
                        put4(at + p * o.g_plane, h, 4);
                        g -= __builtin_convertvector(h, acc4);
                    }
                }
            }
        } else {
            float rest = 0.f;
            const typename T::E* w = nullptr;
            if (o.target_rest && z == 0 && row && counts(o.target[m], o.V)) {
                rest = o.target_rest[m];
                w = static_cast<const typename T::E*>(o.W) + o.target[m] * o.ldw;
            }
#pragma unroll
            for (int j = 0; j < T::TN; ++j) {
                const int64_t n = n_lane + 16 * j;
                if (!row || n >= N)
                    continue;
                if (w) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (n + r < N)
                            acc[i][j][r] = fmaf(rest, static_cast<float>(w[n + r]), acc[i][j][r]);
                }
                if (o.bf16) {
                    put4(static_cast<__bf16*>(o.c) + m * o.ldc + n, __builtin_convertvector(acc[i][j], b4), N - n);
                } else {
                    float* at = static_cast<float*>(o.c) + z * o.split_stride + m * o.ldc + n;
                    acc4 v = acc[i][j];
                    if (o.add) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (n + r < N)
                                v[r] += at[r];
                    }
                    put4(at, v, N - n);
                }
            }
        }
    }
}

// M x N tiles over k split gridDim.y ways (k_split values each, a multiple of
// the step).
template <typename T, Use USE>
__global__ __launch_bounds__(T::NT, 2) void product_kernel(Operand a, Operand b, Parts parts, Out o, int64_t M, int64_t N,
                                                        int64_t K, int64_t k_split, int64_t tiles_m, int64_t tiles_n,
                                                        int group)
{
    int64_t tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, group, tm, tn);
    const int64_t k0 = blockIdx.y * k_split;
    T tile;
    acc4 acc[T::TM][T::TN];
    tile.run(acc, a, b, parts, tm * T::BM, tn * T::BN, k0, K - k0 < k_split ? K - k0 : k_split);
    finish<T, USE>(acc, o, tm * T::BM, tn * T::BN, tn, M, N, static_cast<int>(blockIdx.y));
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

// One wave a row: lse and loss from the tiles' partial runs, each lane taking
// every 64th, then joined across the wave in a fixed order.
__global__ __launch_bounds__(THREADS) void loss_kernel(const Run* __restrict__ part, int64_t nparts,
                                                       const float* __restrict__ target_logit,
                                                       const int64_t* __restrict__ target, int64_t T, int64_t V,
                                                       float* __restrict__ loss, float* __restrict__ lse_out)
{
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (THREADS / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= T)
        return;
    Run r{-INFINITY, 0.f};
    for (int64_t p = lane; p < nparts; p += 64)
        r = join(r, part[row * nparts + p]);
    r = wave_join(r);
    if (lane == 0) {
        const float lse = r.m == -INFINITY && r.s == 0.f ? -INFINITY : r.m + logf(r.s);
        lse_out[row] = lse;
        loss[row] = counts(target[row], V) ? lse - target_logit[row] : 0.f;
    }
}

// The factor form's second step: a workgroup joins its row's runs, then turns
// its share of the row's logits into G, in place and as the operand of dX
// (bf16 or fp32, ldg apart, zeros past V).
constexpr int FACTOR_COLS = 4096;

template <typename E>
__global__ __launch_bounds__(THREADS) void factor_kernel(const Run* __restrict__ part, int64_t nparts,
                                                         const float* __restrict__ target_logit,
                                                         const int64_t* __restrict__ target,
                                                         const float* __restrict__ dloss, int64_t T, int64_t V,
                                                         float* __restrict__ loss, float* __restrict__ U,
                                                         E* __restrict__ g, int64_t ldg,
                                                         float* __restrict__ target_rest)
{
    __shared__ Run runs[THREADS / 64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int64_t row = blockIdx.y; row < T; row += gridDim.y) {
        Run r{-INFINITY, 0.f};
        for (int64_t p = threadIdx.x; p < nparts; p += THREADS)
            r = join(r, part[row * nparts + p]);
        r = wave_join(r);
        __syncthreads();   // the row before has read its runs
        if (lane == 0)
            runs[w] = r;
        __syncthreads();
        r = join(join(runs[0], runs[1]), join(runs[2], runs[3]));
        const float lse = r.m == -INFINITY && r.s == 0.f ? -INFINITY : r.m + logf(r.s);
        const int64_t t = target[row];
        const bool has = counts(t, V);
        const float d = dloss[row];
        if (blockIdx.x == 0 && threadIdx.x == 0)
            loss[row] = has ? lse - target_logit[row] : 0.f;
        const int64_t from = static_cast<int64_t>(blockIdx.x) * FACTOR_COLS;
        for (int64_t v = from + threadIdx.x; v < from + FACTOR_COLS && v < ldg; v += THREADS) {
            float x = 0.f;
            if (v < V) {
                if (has)
                    x = (exp_f(U[row * V + v] - lse) - (v == t ? 1.f : 0.f)) * d;
                U[row * V + v] = x;
            }
            g[row * ldg + v] = static_cast<E>(x);
            if (has && v == t)
                target_rest[row] = x - static_cast<float>(static_cast<E>(x));
        }
    }
}

// A matrix copied with its rows padded to ldo values (zeros), rows without a
// target (where a target list is given) cleared; or split into its exact bf16
// parts h + m + l, planes apart (fp32 input only).
template <typename E, typename O, int PARTS>
__global__ __launch_bounds__(THREADS) void lay_out_kernel(const E* __restrict__ x, int64_t rows, int64_t cols,
                                                          int64_t ldo, const int64_t* __restrict__ target, int64_t V,
                                                          O* __restrict__ out, int64_t plane)
{
    const int64_t per_row = ldo / GROUP, groups = rows * per_row, step = static_cast<int64_t>(gridDim.x) * THREADS;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; q < groups; q += step) {
        const int64_t row = q / per_row, c = (q - row * per_row) * GROUP;
        float v[GROUP];
        load_some(x + row * cols + c, cols - c, v);
        if (target && !counts(target[row], V))
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            store_group(out + p * plane + row * ldo + c, v);
            if (p + 1 < PARTS)
#pragma unroll
                for (int i = 0; i < GROUP; ++i)
                    v[i] -= static_cast<float>(static_cast<__bf16>(v[i]));
        }
    }
}

// The splits' sums in order, rounded once to the result's type.
template <typename O>
__global__ __launch_bounds__(THREADS) void join_splits_kernel(const float* __restrict__ part, int splits,
                                                              int64_t stride, int64_t n, O* __restrict__ out)
{
    const int64_t groups = (n + GROUP - 1) / GROUP, step = static_cast<int64_t>(gridDim.x) * THREADS;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; q < groups; q += step) {
        float v[GROUP], x[GROUP];
        load_some(part + q * GROUP, n - q * GROUP, v);
        for (int s = 1; s < splits; ++s) {
            load_some(part + s * stride + q * GROUP, n - q * GROUP, x);
#pragma unroll
            for (int i = 0; i < GROUP; ++i)
                v[i] += x[i];
        }
        store_some(out + q * GROUP, n - q * GROUP, v);
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

// Tile shapes: 32 rows where there are no more (bound by reading the other
// operand), 256 x 256 (one workgroup a CU) where enough of them fill the GPU,
// else 128 x 128 (two a CU).
template <typename E, bool AK, bool BK>
using Thin = Tile<E, AK, BK, 32, 64, 32, 16, 4>;
template <typename E, bool AK, bool BK>
using Square = Tile<E, AK, BK, 128, 128, 64, 64, 2>;
template <typename E, bool AK, bool BK>
using Large = Tile<E, AK, BK, 256, 256, 128, 64, 2>;

enum ShapeKind { THIN, SQUARE, LARGE };

struct Shape {
    ShapeKind kind;
    int64_t bm, bn, waves_n;
};

template <typename E>
Shape shape_for(int64_t M, int64_t N)
{
    if (M <= 32)
        return Shape{THIN, 32, 64, 4};
    if (sizeof(E) == 2) {
        const int64_t cus = device_cu_count();
        const int64_t large = ceil_div(ceil_div(M, 256) * ceil_div(N, 256), cus) * 4;
        const int64_t square = ceil_div(ceil_div(M, 128) * ceil_div(N, 128), 2 * cus) * 2;
        if (4 * large <= 5 * square)
            return Shape{LARGE, 256, 256, 4};
    }
    return Shape{SQUARE, 128, 128, 2};
}

template <typename E>
int64_t parts_of(int64_t M, int64_t N)
{
    const Shape s = shape_for<E>(M, N);
    return ceil_div(N, s.bn) * s.waves_n;
}

// How many ways to split k so that the tiles fill the GPU: about two
// workgroups a CU, at least eight steps each.
template <typename E>
int64_t splits_for(int64_t M, int64_t N, int64_t K)
{
    const Shape s = shape_for<E>(M, N);
    const int64_t step = STEP_BYTES / sizeof(E);
    const int64_t tiles = ceil_div(M, s.bm) * ceil_div(N, s.bn), steps = ceil_div(K, step);
    return std::max<int64_t>(1, std::min<int64_t>(2 * device_cu_count() / std::max<int64_t>(tiles, 1), steps / 8));
}

template <typename T, Use USE>
hipError_t launch_product(const Operand& a, const Operand& b, const Parts& p, const Out& o, int64_t M, int64_t N,
                          int64_t K, int64_t splits, hipStream_t s)
{
    const int64_t tm = ceil_div(M, T::BM), tn = ceil_div(N, T::BN);
    const int64_t k_split = round_up(ceil_div(std::max<int64_t>(K, 1), splits), T::STEP);
    product_kernel<T, USE><<<dim3(static_cast<unsigned>(tm * tn), static_cast<unsigned>(splits)), T::NT, 0, s>>>(
        a, b, p, o, M, N, K, k_split, tm, tn, 1024 / T::BM);
    return hipGetLastError();
}

template <typename E, bool AK, bool BK, Use USE>
hipError_t product(const Operand& a, const Operand& b, const Parts& p, const Out& o, int64_t M, int64_t N, int64_t K,
                   int64_t splits, hipStream_t s)
{
    const ShapeKind kind = shape_for<E>(M, N).kind;
    if (kind == THIN)
        return launch_product<Thin<E, AK, BK>, USE>(a, b, p, o, M, N, K, splits, s);
    if constexpr (sizeof(E) == 2)
        if (kind == LARGE)
            return launch_product<Large<E, AK, BK>, USE>(a, b, p, o, M, N, K, splits, s);
    return launch_product<Square<E, AK, BK>, USE>(a, b, p, o, M, N, K, splits, s);
}

constexpr Parts ONE{1, 0};
constexpr Parts THREE_A{3, 0x210};   // A in three parts, B in one

template <typename O>
hipError_t join_splits(const float* part, int64_t splits, int64_t n, O* out, hipStream_t s)
{
    join_splits_kernel<O><<<grid_for(ceil_div(n, THREADS * GROUP)), THREADS, 0, s>>>(part, static_cast<int>(splits), n,
                                                                                     n, out);
    return hipGetLastError();
}

// X or W as an operand: as it is where its rows lie on 16-byte boundaries,
// else a copy with padded rows (and, given targets, the rows without one
// cleared).
template <typename E>
bool needs_copy(const void* p, int64_t D)
{
    return !aligned16(p) || D * static_cast<int64_t>(sizeof(E)) % 16 != 0;
}

template <typename E>
hipError_t copy_rows(const E* x, int64_t rows, int64_t D, int64_t ldo, const int64_t* target, int64_t V, E* out,
                     hipStream_t s)
{
    lay_out_kernel<E, E, 1><<<grid_for(ceil_div(rows * (ldo / GROUP), THREADS)), THREADS, 0, s>>>(x, rows, D, ldo,
                                                                                               target, V, out, 0);
    return hipGetLastError();
}

// Arrays of a call in its workspace; sized with a null base.
constexpr int64_t PIECE_BYTES = int64_t(512) << 20;   // of G at a time

struct Plan {
    int64_t ldd = 0;                      // row length of copies
    void* x = nullptr;
    void* w = nullptr;
    Run* part = nullptr;
    int64_t nparts = 0;
    float* target_logit = nullptr;
    void* g = nullptr;
    int64_t piece = 0, ldg = 0, g_parts = 0, dx_splits = 1, dw_splits = 1;
    float* target_rest = nullptr;
    float* dx = nullptr;
    float* dw = nullptr;
    int64_t bytes = 0;
};

template <typename E>
Plan make_plan(int op, int64_t T, int64_t V, int64_t D, bool copy_x, bool copy_w, char* base)
{
    constexpr int64_t SZ = sizeof(E);
    Plan p;
    Arena a{base};
    p.ldd = round_up(D, GROUP);
    if (op == POSEIDON_XENT_BACKWARD || copy_x)
        p.x = a.take(T * p.ldd * SZ);
    if (copy_w)
        p.w = a.take(V * p.ldd * SZ);
    if (op != POSEIDON_XENT_BACKWARD) {
        p.nparts = parts_of<E>(T, V);
        p.part = static_cast<Run*>(a.take(T * p.nparts * sizeof(Run)));
        p.target_logit = static_cast<float*>(a.take(T * 4));
    }
    if (op == POSEIDON_XENT_FORWARD) {
        p.bytes = a.at;
        return p;
    }
    p.g_parts = SZ == 4 ? 0 : op == POSEIDON_XENT_BACKWARD ? 3 : 1;
    const int64_t g_value = SZ == 4 ? 4 : 2 * p.g_parts;
    p.piece = round_up(V, GROUP);
    if (op == POSEIDON_XENT_BACKWARD)
        p.piece = std::min(p.piece, std::max<int64_t>(PIECE_BYTES / g_value / std::max<int64_t>(T, 1) / 256, 1) * 256);
    p.ldg = p.piece;
    p.g = a.take(T * p.ldg * g_value);
    p.target_rest = static_cast<float*>(a.take(T * 4));
    p.dx_splits = splits_for<E>(T, D, std::min(p.piece, V));
    const int64_t pieces = ceil_div(V, p.piece);
    if (p.dx_splits > 1 || (pieces > 1 && SZ == 2))
        p.dx = static_cast<float*>(a.take(p.dx_splits * T * D * 4));
    if (op == POSEIDON_XENT_BACKWARD) {
        p.dw_splits = splits_for<E>(std::min(p.piece, V), D, T);
        if (p.dw_splits > 1)
            p.dw = static_cast<float*>(a.take(p.dw_splits * std::min(p.piece, V) * D * 4));
    }
    p.bytes = a.at;
    return p;
}

#define POSEIDON_TRY(x)              \
    do {                             \
        const hipError_t rc_ = (x);  \
        if (rc_ != hipSuccess)       \
            return rc_;              \
    } while (0)

template <typename E>
hipError_t forward_typed(const E* X, const E* W, const int64_t* target, int64_t T, int64_t V, int64_t D, float* loss,
                         float* lse, char* ws, hipStream_t s)
{
    const bool cx = needs_copy<E>(X, D), cw = needs_copy<E>(W, D);
    const Plan p = make_plan<E>(POSEIDON_XENT_FORWARD, T, V, D, cx, cw, ws);
    if (cx)
        POSEIDON_TRY(copy_rows(X, T, D, p.ldd, nullptr, V, static_cast<E*>(p.x), s));
    if (cw)
        POSEIDON_TRY(copy_rows(W, V, D, p.ldd, nullptr, V, static_cast<E*>(p.w), s));
    Out o{};
    o.part = p.part;
    o.nparts = p.nparts;
    o.target_logit = p.target_logit;
    o.target = target;
    const Operand a{cx ? p.x : X, cx ? p.ldd : D, T, 0}, b{cw ? p.w : W, cw ? p.ldd : D, V, 0};
    POSEIDON_TRY((product<E, true, true, STATS>(a, b, ONE, o, T, V, round_up(D, 16 / sizeof(E)), 1, s)));
    loss_kernel<<<static_cast<unsigned>(ceil_div(T, THREADS / 64)), THREADS, 0, s>>>(p.part, p.nparts, p.target_logit,
                                                                                    target, T, V, loss, lse);
    return hipGetLastError();
}

// dX = G W for one piece of the vocabulary (the first replaces, the others add).
template <typename E>
hipError_t input_gradient(const Plan& p, const Operand& g, const Operand& w, const E* W, const int64_t* target,
                          int64_t T, int64_t V, int64_t D, int64_t v0, int64_t vp, E* dX, hipStream_t s)
{
    const bool first = v0 == 0, last = v0 + vp == V;
    constexpr bool BF16 = sizeof(E) == 2;
    Out o{};
    o.c = p.dx ? static_cast<void*>(p.dx) : static_cast<void*>(dX);
    o.ldc = D;
    o.split_stride = T * D;
    o.bf16 = BF16 && !p.dx;
    o.add = !first;
    if (BF16 && last) {   // every piece has left its targets' rest by now
        o.target_rest = p.target_rest;
        o.target = target;
        o.V = V;
        o.W = W;
        o.ldw = w.ld;
    }
    POSEIDON_TRY((product<E, true, false, STORE>(g, w, ONE, o, T, D, round_up(vp, GROUP), p.dx_splits, s)));
    return last && p.dx ? join_splits(p.dx, p.dx_splits, T * D, dX, s) : hipSuccess;
}

template <typename E>
hipError_t backward_typed(const E* X, const E* W, const int64_t* target, const float* lse, const float* dloss,
                          int64_t T, int64_t V, int64_t D, E* dX, float* dW, char* ws, hipStream_t s)
{
    const bool cw = needs_copy<E>(W, D);
    const Plan p = make_plan<E>(POSEIDON_XENT_BACKWARD, T, V, D, true, cw, ws);
    // X without the rows that have no target: whatever they hold must not
    // reach dW.
    if (T > 0)
        POSEIDON_TRY(copy_rows(X, T, D, p.ldd, target, V, static_cast<E*>(p.x), s));
    if (cw)
        POSEIDON_TRY(copy_rows(W, V, D, p.ldd, nullptr, V, static_cast<E*>(p.w), s));
    const E* w = cw ? static_cast<const E*>(p.w) : W;
    const int64_t ldw = cw ? p.ldd : D;
    const Operand x{p.x, p.ldd, T, 0};
    for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
        const int64_t vp = std::min(p.piece, V - v0);
        const Operand wp{w + v0 * ldw, ldw, vp, 0};
        const Operand g{p.g, p.ldg, T, T * p.ldg};
        if (T > 0) {
            Out o{};
            o.target = target;
            o.lse = lse;
            o.dloss = dloss;
            o.g = p.g;
            o.ldg = p.ldg;
            o.g_plane = T * p.ldg;
            o.g_parts = static_cast<int32_t>(p.g_parts);
            o.v0 = v0;
            o.V = V;
            o.target_rest = sizeof(E) == 2 ? p.target_rest : nullptr;
            POSEIDON_TRY((product<E, true, true, GRAD>(x, wp, ONE, o, T, vp, round_up(D, 16 / sizeof(E)), 1, s)));
            POSEIDON_TRY(input_gradient(p, g, wp, w, target, T, V, D, v0, vp, dX, s));
        }
        Out o{};
        o.c = p.dw ? p.dw : dW + v0 * D;
        o.ldc = D;
        o.split_stride = vp * D;
        POSEIDON_TRY((product<E, false, false, STORE>(g, x, p.g_parts == 3 ? THREE_A : ONE, o, vp, D, T, p.dw_splits,
                                                      s)));
        if (p.dw)
            POSEIDON_TRY(join_splits(p.dw, p.dw_splits, vp * D, dW + v0 * D, s));
    }
    return hipSuccess;
}

template <typename E>
hipError_t factor_typed(const E* X, const E* W, const int64_t* target, const float* dloss, int64_t T, int64_t V,
                        int64_t D, float* loss, float* U, E* dX, char* ws, hipStream_t s)
{
    const bool cx = needs_copy<E>(X, D), cw = needs_copy<E>(W, D);
    const Plan p = make_plan<E>(POSEIDON_XENT_FACTOR, T, V, D, cx, cw, ws);
    if (cx)
        POSEIDON_TRY(copy_rows(X, T, D, p.ldd, nullptr, V, static_cast<E*>(p.x), s));
    if (cw)
        POSEIDON_TRY(copy_rows(W, V, D, p.ldd, nullptr, V, static_cast<E*>(p.w), s));
    Out o{};
    o.part = p.part;
    o.nparts = p.nparts;
    o.target_logit = p.target_logit;
    o.target = target;
    o.c = U;
    o.ldc = V;
    const Operand a{cx ? p.x : X, cx ? p.ldd : D, T, 0}, b{cw ? p.w : W, cw ? p.ldd : D, V, 0};
    POSEIDON_TRY((product<E, true, true, LOGITS>(a, b, ONE, o, T, V, round_up(D, 16 / sizeof(E)), 1, s)));
    const dim3 grid(static_cast<unsigned>(ceil_div(p.ldg, FACTOR_COLS)), static_cast<unsigned>(std::min<int64_t>(T, 32768)));
    factor_kernel<E><<<grid, THREADS, 0, s>>>(p.part, p.nparts, p.target_logit, target, dloss, T, V, loss, U,
                                              static_cast<E*>(p.g), p.ldg, p.target_rest);
    POSEIDON_TRY(hipGetLastError());
    return input_gradient(p, Operand{p.g, p.ldg, T, 0}, b, static_cast<const E*>(b.p), target, T, V, D, 0, V, dX, s);
}

}  // namespace

int64_t xent_workspace(int32_t op, const void* X, const void* W, int64_t T, int64_t V, int64_t D, int32_t dtype)
{
    return dtype == POSEIDON_BF16
               ? make_plan<__bf16>(op, T, V, D, needs_copy<__bf16>(X, D), needs_copy<__bf16>(W, D), nullptr).bytes
               : make_plan<float>(op, T, V, D, needs_copy<float>(X, D), needs_copy<float>(W, D), nullptr).bytes;
}

hipError_t launch_xent_forward(const void* X, const void* W, const int64_t* target, int64_t T, int64_t V, int64_t D,
                               int32_t dtype, float* loss, float* lse, void* ws, hipStream_t stream)
{
    char* w = static_cast<char*>(ws);
    if (dtype == POSEIDON_BF16)
        return forward_typed(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W), target, T, V, D, loss, lse,
                             w, stream);
    return forward_typed(static_cast<const float*>(X), static_cast<const float*>(W), target, T, V, D, loss, lse, w,
                         stream);
}

hipError_t launch_xent_backward(const void* X, const void* W, const int64_t* target, const float* lse,
                                const float* dloss, int64_t T, int64_t V, int64_t D, int32_t dtype, void* dX,
                                float* dW, void* ws, hipStream_t stream)
{
    char* w = static_cast<char*>(ws);
    if (dtype == POSEIDON_BF16)
        return backward_typed(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W), target, lse, dloss, T, V,
                              D, static_cast<__bf16*>(dX), dW, w, stream);
    return backward_typed(static_cast<const float*>(X), static_cast<const float*>(W), target, lse, dloss, T, V, D,
                          static_cast<float*>(dX), dW, w, stream);
}

hipError_t launch_xent_factor(const void* X, const void* W, const int64_t* target, const float* dloss, int64_t T,
                              int64_t V, int64_t D, int32_t dtype, float* loss, float* U, void* dX, void* ws,
                              hipStream_t stream)
{
    char* w = static_cast<char*>(ws);
    if (dtype == POSEIDON_BF16)
        return factor_typed(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W), target, dloss, T, V, D, loss,
                            U, static_cast<__bf16*>(dX), w, stream);
    return factor_typed(static_cast<const float*>(X), static_cast<const float*>(W), target, dloss, T, V, D, loss, U,
                        static_cast<float*>(dX), w, stream);
}

}  // namespace poseidon
