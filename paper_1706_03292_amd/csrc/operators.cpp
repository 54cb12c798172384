// The C entry points of the operators at a network's end (include/poseidon.h):
// the argument checks, then the launchers of norm.hip and xent.hip.  Host code
// only; every check runs before anything is enqueued.
#include <math.h>

#include "common.h"

namespace poseidon {
namespace {

// Bytes of a value, or 0 for an unknown type.
int64_t size_of(int32_t dtype) { return dtype == POSEIDON_F32 ? 4 : dtype == POSEIDON_BF16 ? 2 : 0; }

// rows x cols values of up to 4 bytes, addressable and not negative.
bool sizes_ok(int64_t rows, int64_t cols)
{
    return rows >= 0 && cols >= 0 && (cols == 0 || rows <= INT64_MAX / 16 / cols);
}

// p as the 16-bit threshold of the mask, or -1.
int32_t threshold(double p) { return p >= 0.0 && p <= 1.0 ? static_cast<int32_t>(floor(p * 65536.0 + 0.5)) : -1; }

// The ranges a call reads and writes: whether a written one overlaps another
// or a read one.  A fixed number of them, so that nothing here can throw.
struct Ranges {
    Span reads[8], writes[8];
    int nr = 0, nw = 0;
    static void add(Span (&v)[8], int& n, const void* p, int64_t bytes)
    {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        if (p && bytes > 0 && n < 8)
            v[n++] = Span{lo, lo + static_cast<uintptr_t>(bytes)};
    }
    void in(const void* p, int64_t bytes) { add(reads, nr, p, bytes); }
    void out(const void* p, int64_t bytes) { add(writes, nw, p, bytes); }
    static bool meet(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }
    bool collide() const
    {
        for (int i = 0; i < nw; ++i) {
            for (int j = 0; j < nr; ++j)
                if (meet(writes[i], reads[j]))
                    return true;
            for (int j = 0; j < i; ++j)
                if (meet(writes[i], writes[j]))
                    return true;
        }
        return false;
    }
};

int status(hipError_t rc) { return rc == hipSuccess ? POSEIDON_OK : POSEIDON_ERR_HIP; }

constexpr int64_t MOST_COLS = int64_t(1) << 28;
// A tile's 256 rows of W, X or G lie within the 2 GB that one buffer resource
// addresses.
constexpr int64_t MOST_ROWS = int64_t(1) << 24, MOST_CLASSES = int64_t(1) << 21, MOST_FEATURES = int64_t(1) << 20;
constexpr int64_t MOST_LOGITS = int64_t(1) << 37;

bool xent_sizes_ok(int64_t T, int64_t V, int64_t D, int32_t dtype)
{
    return size_of(dtype) && T >= 0 && T <= MOST_ROWS && V >= 1 && V <= MOST_CLASSES && D >= 1 && D <= MOST_FEATURES &&
           T * V <= MOST_LOGITS;
}

bool workspace_ok(const void* ws, int64_t bytes, int64_t needed)
{
    return needed == 0 || (ws && aligned16(ws) && bytes >= needed);
}

}  // namespace
}  // namespace poseidon

using namespace poseidon;

extern "C" int poseidon_dropout(const void* x, const void* residual, int64_t rows, int64_t cols, int32_t dtype,
                                double p, const int64_t* rng, void* y, hipStream_t stream)
{
    const int64_t size = size_of(dtype);
    const int32_t thr = threshold(p);
    if (!size || !sizes_ok(rows, cols) || thr < 0)
        return POSEIDON_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0)
        return POSEIDON_OK;
    if (!x || !y || (thr && !rng))
        return POSEIDON_ERR_INVALID_ARG;
    Ranges r;
    r.in(x, rows * cols * size);
    r.in(residual, rows * cols * size);
    r.in(thr ? rng : nullptr, 16);
    r.out(y, rows * cols * size);
    if (r.collide())
        return POSEIDON_ERR_INVALID_ARG;
    return status(launch_dropout(x, residual, rows, cols, dtype, static_cast<uint32_t>(thr), rng, y, stream));
}

extern "C" int poseidon_norm_forward(const void* x, const void* residual, const float* gamma, const float* beta,
                                     int64_t rows, int64_t cols, int32_t dtype, float eps, double p,
                                     const int64_t* rng, void* h, void* y, float* mean, float* rstd,
                                     hipStream_t stream)
{
    const int64_t size = size_of(dtype);
    const int32_t thr = threshold(p);
    if (!size || !sizes_ok(rows, cols) || cols > MOST_COLS || thr < 0 || !(eps >= 0.f))
        return POSEIDON_ERR_INVALID_ARG;
    if (rows == 0)
        return POSEIDON_OK;
    if (cols < 1 || !x || !gamma || !beta || !y || !mean || !rstd || (thr && !rng))
        return POSEIDON_ERR_INVALID_ARG;
    Ranges r;
    r.in(x, rows * cols * size);
    r.in(residual, rows * cols * size);
    r.in(gamma, cols * 4);
    r.in(beta, cols * 4);
    r.in(thr ? rng : nullptr, 16);
    r.out(h, rows * cols * size);
    r.out(y, rows * cols * size);
    r.out(mean, rows * 4);
    r.out(rstd, rows * 4);
    if (r.collide())
        return POSEIDON_ERR_INVALID_ARG;
    return status(launch_norm_forward(x, residual, gamma, beta, rows, cols, dtype, eps, static_cast<uint32_t>(thr),
                                      rng, h, y, mean, rstd, stream));
}

extern "C" int poseidon_norm_workspace(int64_t rows, int64_t cols, int64_t* bytes)
{
    if (!bytes || !sizes_ok(rows, cols) || cols > MOST_COLS)
        return POSEIDON_ERR_INVALID_ARG;
    *bytes = cols == 0 ? 0 : norm_backward_workspace(rows, cols);
    return POSEIDON_OK;
}

extern "C" int poseidon_norm_backward(const void* dy, const void* h, const float* gamma, const float* mean,
                                      const float* rstd, const void* dresidual, int64_t rows, int64_t cols,
                                      int32_t dtype, double p, const int64_t* rng, void* dx, void* dh, float* dgamma,
                                      float* dbeta, void* workspace, int64_t workspace_bytes, hipStream_t stream)
{
    const int64_t size = size_of(dtype);
    int32_t thr = threshold(p);
    if (!size || !sizes_ok(rows, cols) || cols > MOST_COLS || thr < 0)
        return POSEIDON_ERR_INVALID_ARG;
    if (rows == 0)
        thr = 0;   // a launch still clears dgamma and dbeta: without rows nothing is dropped, and no rng is read
    if (cols < 1)
        return rows == 0 ? POSEIDON_OK : POSEIDON_ERR_INVALID_ARG;
    if (!dgamma || !dbeta || (rows > 0 && (!dy || !h || !gamma || !mean || !rstd || !dh || (thr && (!rng || !dx)))))
        return POSEIDON_ERR_INVALID_ARG;
    const int64_t needed = norm_backward_workspace(rows, cols);
    if (!workspace_ok(workspace, workspace_bytes, needed))
        return POSEIDON_ERR_INVALID_ARG;
    Ranges r;
    r.in(dy, rows * cols * size);
    r.in(h, rows * cols * size);
    r.in(gamma, cols * 4);
    r.in(mean, rows * 4);
    r.in(rstd, rows * 4);
    r.in(dresidual, rows * cols * size);
    r.in(thr ? rng : nullptr, 16);
    r.out(thr ? dx : nullptr, rows * cols * size);
    r.out(dh, rows * cols * size);
    r.out(dgamma, cols * 4);
    r.out(dbeta, cols * 4);
    r.out(workspace, needed);
    if (r.collide())
        return POSEIDON_ERR_INVALID_ARG;
    return status(launch_norm_backward(dy, h, gamma, mean, rstd, dresidual, rows, cols, dtype,
                                       static_cast<uint32_t>(thr), rng, dx, dh, dgamma, dbeta, workspace, stream));
}

extern "C" int poseidon_xent_workspace(int32_t op, const void* X, const void* W, int64_t T, int64_t V, int64_t D,
                                       int32_t dtype, int64_t* bytes)
{
    if (!bytes || op < POSEIDON_XENT_FORWARD || op > POSEIDON_XENT_FACTOR || !xent_sizes_ok(T, V, D, dtype))
        return POSEIDON_ERR_INVALID_ARG;
    *bytes = xent_workspace(op, X, W, T, V, D, dtype);
    return POSEIDON_OK;
}

extern "C" int poseidon_xent_forward(const void* X, const void* W, const int64_t* target, int64_t T, int64_t V,
                                     int64_t D, int32_t dtype, float* loss, float* lse, void* workspace,
                                     int64_t workspace_bytes, hipStream_t stream)
{
    if (!xent_sizes_ok(T, V, D, dtype))
        return POSEIDON_ERR_INVALID_ARG;
    if (T == 0)
        return POSEIDON_OK;
    const int64_t size = size_of(dtype), needed = xent_workspace(POSEIDON_XENT_FORWARD, X, W, T, V, D, dtype);
    if (!X || !W || !target || !loss || !lse || !workspace_ok(workspace, workspace_bytes, needed))
        return POSEIDON_ERR_INVALID_ARG;
    Ranges r;
    r.in(X, T * D * size);
    r.in(W, V * D * size);
    r.in(target, T * 8);
    r.out(loss, T * 4);
    r.out(lse, T * 4);
    r.out(workspace, needed);
    if (r.collide())
        return POSEIDON_ERR_INVALID_ARG;
    return status(launch_xent_forward(X, W, target, T, V, D, dtype, loss, lse, workspace, stream));
}

extern "C" int poseidon_xent_backward(const void* X, const void* W, const int64_t* target, const float* lse,
                                      const float* dloss, int64_t T, int64_t V, int64_t D, int32_t dtype, void* dX,
                                      float* dW, void* workspace, int64_t workspace_bytes, hipStream_t stream)
{
    if (!xent_sizes_ok(T, V, D, dtype))
        return POSEIDON_ERR_INVALID_ARG;
    const int64_t size = size_of(dtype), needed = xent_workspace(POSEIDON_XENT_BACKWARD, X, W, T, V, D, dtype);
    if (!W || !dW || (T > 0 && (!X || !target || !lse || !dloss || !dX)) ||
        !workspace_ok(workspace, workspace_bytes, needed))
        return POSEIDON_ERR_INVALID_ARG;
    Ranges r;
    r.in(X, T * D * size);
    r.in(W, V * D * size);
    r.in(target, T * 8);
    r.in(lse, T * 4);
    r.in(dloss, T * 4);
    r.out(dX, T * D * size);
    r.out(dW, V * D * 4);
    r.out(workspace, needed);
    if (r.collide())
        return POSEIDON_ERR_INVALID_ARG;
    return status(launch_xent_backward(X, W, target, lse, dloss, T, V, D, dtype, dX, dW, workspace, stream));
}

extern "C" int poseidon_xent_factor(const void* X, const void* W, const int64_t* target, const float* dloss,
                                    int64_t T, int64_t V, int64_t D, int32_t dtype, float* loss, float* U, void* dX,
                                    void* workspace, int64_t workspace_bytes, hipStream_t stream)
{
    if (!xent_sizes_ok(T, V, D, dtype))
        return POSEIDON_ERR_INVALID_ARG;
    if (T == 0)
        return POSEIDON_OK;
    const int64_t size = size_of(dtype), needed = xent_workspace(POSEIDON_XENT_FACTOR, X, W, T, V, D, dtype);
    if (!X || !W || !target || !dloss || !loss || !U || !dX || !workspace_ok(workspace, workspace_bytes, needed))
        return POSEIDON_ERR_INVALID_ARG;
    Ranges r;
    r.in(X, T * D * size);
    r.in(W, V * D * size);
    r.in(target, T * 8);
    r.in(dloss, T * 4);
    r.out(loss, T * 4);
    r.out(U, T * V * 4);
    r.out(dX, T * D * size);
    r.out(workspace, needed);
    if (r.collide())
        return POSEIDON_ERR_INVALID_ARG;
    return status(launch_xent_factor(X, W, target, dloss, T, V, D, dtype, loss, U, dX, workspace, stream));
}
