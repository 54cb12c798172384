// The optimizer object of poseidon_adamw_* (include/poseidon.h): the argument
// checks, the tensors in launches of up to ADAMW_GROUP, then the launchers of
// adamw.hip.  Host code only; every check runs before anything is enqueued, and
// no exception leaves an entry point.
#include <math.h>

#include <new>

#include "optimizer.h"

struct poseidon_adamw {
    std::vector<poseidon_adamw_tensor> tensors;   // all of them, the empty ones too
    std::vector<int64_t> first_group;
    std::vector<poseidon::Span> reads, writes;    // of all calls, sorted and disjoint
    // what a step launches from the shards and from the sums, by kind (kind_of)
    std::vector<poseidon::AdamwGroup> steps[4], sum_steps[4];
    std::vector<poseidon::AdamwGroup> squares[2]; // what a clip launches: several rows of gradients, one
    int64_t chunk = 0;                            // values of a clip's workgroup
    int64_t parts = 0;                            // its workgroups
    int32_t dtype = 0;
    bool sums = true;                             // every tensor with values has a sum
};

namespace poseidon {
namespace {

constexpr int64_t MOST_VALUES = int64_t(1) << 34, MOST_STRIDE = int64_t(1) << 56;
constexpr int32_t MOST_WORKERS = 1024;
// Workgroups of a clip: enough loads in flight, few enough partial sums that adding
// them costs little (VGG19-22K's 229M values, fp32: 2048 of them 177 us, 4096 154, 8192
// 142, 32768 148).
constexpr int64_t CLIP_BLOCKS = 8192;

int64_t value_size(int32_t dtype) { return dtype == POSEIDON_BF16 ? 2 : 4; }
int64_t blocks_of(int64_t n, int64_t chunk) { return (n + chunk - 1) / chunk; }
int status(hipError_t rc) { return rc == hipSuccess ? POSEIDON_OK : POSEIDON_ERR_HIP; }

bool tensor_ok(const poseidon_adamw_tensor& t)
{
    if (t.n < 0 || t.n > MOST_VALUES || t.P < 1 || t.P > MOST_WORKERS || !(t.weight_decay >= 0.f) ||
        !isfinite(t.weight_decay))
        return false;
    if (t.n == 0)
        return true;
    return t.W && t.shards && t.m && t.v && (t.P == 1 || (t.stride >= t.n && t.stride <= MOST_STRIDE / t.P));
}

void add(std::vector<AdamwGroup>& to, const AdamwItem& item, int64_t chunk)
{
    const int64_t blocks = blocks_of(item.n, chunk);
    if (to.empty() || to.back().count == ADAMW_GROUP || to.back().blocks + blocks > ADAMW_MOST_BLOCKS) {
        to.emplace_back();
        AdamwGroup& g = to.back();
        g.count = g.blocks = 0;
        g.chunk = chunk;
        std::fill(g.first_block, g.first_block + ADAMW_GROUP, INT32_MAX);
    }
    AdamwGroup& g = to.back();
    g.first_block[g.count] = g.blocks;
    g.item[g.count++] = item;
    g.blocks += static_cast<int32_t>(blocks);
}

AdamwItem item_of(const poseidon_adamw_tensor& t, int64_t first_group)
{
    return AdamwItem{t.W, t.shards, t.m, t.v, t.exponents, t.copy, t.n, t.P > 1 ? t.stride : 0, first_group, t.P,
                     t.weight_decay};
}

// The ranges sorted, those that touch made one.
void merge(std::vector<Span>& v)
{
    std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    size_t n = 0;
    for (const Span& s : v) {
        if (n > 0 && s.lo <= v[n - 1].hi)
            v[n - 1].hi = std::max(v[n - 1].hi, s.hi);
        else
            v[n++] = s;
    }
    v.resize(n);
}

// A step's launches by what their tensors have in common.
int kind_of(const poseidon_adamw_tensor& t, bool one) { return 2 * (t.exponents != nullptr) + one; }

// Whether [p, p + bytes) meets one of the sorted, disjoint ranges.
bool meets(const std::vector<Span>& sorted, const void* p, int64_t bytes)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p), hi = lo + static_cast<uintptr_t>(bytes);
    if (!p || bytes <= 0)
        return false;
    auto it = std::lower_bound(sorted.begin(), sorted.end(), hi, [](const Span& w, uintptr_t h) { return w.lo < h; });
    return it != sorted.begin() && std::prev(it)->hi > lo;
}

int create(const poseidon_adamw_tensor* tensors, int32_t count, int32_t dtype, poseidon_adamw& o)
{
    o.dtype = dtype;
    int64_t total = 0, group = 0;
    for (int32_t i = 0; i < count; ++i) {
        const poseidon_adamw_tensor& t = tensors[i];
        if (!tensor_ok(t))
            return POSEIDON_ERR_INVALID_ARG;
        o.tensors.push_back(t);
        o.first_group.push_back(group);
        if (t.n == 0)
            continue;
        const int64_t moments = t.exponents ? t.n : 4 * t.n;
        total += t.n;
        group += blocks_of(t.n, ADAMW_BLOCK) * (ADAMW_BLOCK / 8);
        for (int64_t p = 0; p < t.P; ++p)
            add_span(o.reads, static_cast<const char*>(t.shards) + (p ? p * t.stride : 0) * value_size(dtype),
                     t.n * value_size(dtype));
        add_span(o.writes, t.W, 4 * t.n);
        add_span(o.writes, t.m, moments);
        add_span(o.writes, t.v, moments);
        add_span(o.writes, t.exponents, 2 * blocks_of(t.n, ADAMW_BLOCK));
        add_span(o.writes, t.copy, 2 * t.n);
        add_span(o.writes, t.sum, 4 * t.n);
        o.sums = o.sums && t.sum;
    }
    if (writes_collide(o.writes, o.reads))
        return POSEIDON_ERR_INVALID_ARG;
    merge(o.writes);
    merge(o.reads);
    o.chunk = std::max<int64_t>(1, blocks_of(blocks_of(total, CLIP_BLOCKS), ADAMW_CHUNK)) * ADAMW_CHUNK;
    for (int32_t i = 0; i < count; ++i) {
        const poseidon_adamw_tensor& t = tensors[i];
        if (t.n == 0)
            continue;
        AdamwItem item = item_of(t, o.first_group[i]);
        add(o.steps[kind_of(t, t.P == 1)], item, ADAMW_CHUNK);
        AdamwItem square = item;
        square.copy = t.sum;
        add(o.squares[t.P == 1], square, o.chunk);
        o.parts += blocks_of(t.n, o.chunk);
        if (o.sums) {
            item.G = t.sum;
            item.stride = 0;
            item.P = 1;
            add(o.sum_steps[kind_of(t, true)], item, ADAMW_CHUNK);
        }
    }
    return POSEIDON_OK;
}

int step(const poseidon_adamw& o, const poseidon_adamw_rule& r, hipStream_t stream)
{
    const int32_t dtype = r.from_sums ? POSEIDON_F32 : o.dtype;
    for (int kind = 0; kind < 4; ++kind)
        for (const AdamwGroup& g : (r.from_sums ? o.sum_steps : o.steps)[kind])
            if (launch_adamw_step(g, dtype, AdamwKind{(kind & 2) != 0, (kind & 1) != 0}, r, stream) != hipSuccess)
                return POSEIDON_ERR_HIP;
    return POSEIDON_OK;
}

int values(const poseidon_adamw& o, float* const* m, float* const* v, hipStream_t stream)
{
    std::vector<AdamwGroup> groups;
    std::vector<Span> out;
    for (size_t i = 0; i < o.tensors.size(); ++i) {
        const poseidon_adamw_tensor& t = o.tensors[i];
        if (t.n == 0 || (!m[i] && !v[i]))
            continue;
        AdamwItem item = item_of(t, 0);
        item.W = m[i];
        item.copy = v[i];
        add(groups, item, ADAMW_CHUNK);
        add_span(out, m[i], 4 * t.n);
        add_span(out, v[i], 4 * t.n);
    }
    std::vector<Span> kept = o.reads;
    kept.insert(kept.end(), o.writes.begin(), o.writes.end());
    if (writes_collide(std::move(out), kept))
        return POSEIDON_ERR_INVALID_ARG;
    for (const AdamwGroup& g : groups)
        if (launch_adamw_values(g, stream) != hipSuccess)
            return POSEIDON_ERR_HIP;
    return POSEIDON_OK;
}

bool beta_ok(double b) { return b >= 0.0 && b < 1.0; }

}  // namespace
}  // namespace poseidon

using namespace poseidon;

extern "C" int poseidon_adamw_create(const poseidon_adamw_tensor* tensors, int32_t count, int32_t dtype,
                                     poseidon_adamw** out)
{
    if (!out)
        return POSEIDON_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 0 || (count > 0 && !tensors) || (dtype != POSEIDON_F32 && dtype != POSEIDON_BF16))
        return POSEIDON_ERR_INVALID_ARG;
    poseidon_adamw* o = new (std::nothrow) poseidon_adamw;
    if (!o)
        return POSEIDON_ERR_HIP;
    int rc = POSEIDON_ERR_HIP;
    try {
        rc = create(tensors, count, dtype, *o);
    } catch (...) {
    }
    if (rc == POSEIDON_OK)
        *out = o;
    else
        delete o;
    return rc;
}

extern "C" int poseidon_adamw_destroy(poseidon_adamw* optimizer)
{
    delete optimizer;
    return POSEIDON_OK;
}

extern "C" int poseidon_adamw_step(const poseidon_adamw* optimizer, const poseidon_adamw_rule* rule,
                                   hipStream_t stream)
{
    if (!optimizer || !rule || rule->reserved != 0)
        return POSEIDON_ERR_INVALID_ARG;
    const poseidon_adamw_rule& r = *rule;
    if ((!r.clock && (!isfinite(r.lr) || r.step < 1)) || !beta_ok(r.beta1) || !beta_ok(r.beta2) ||
        !(static_cast<float>(r.eps) > 0.f) || !isfinite(static_cast<float>(r.eps)) ||
        (r.from_sums != 0 && !(r.from_sums == 1 && optimizer->sums)))
        return POSEIDON_ERR_INVALID_ARG;
    if (meets(optimizer->writes, r.clock, 16) || meets(optimizer->writes, r.scale, 4) ||
        meets(optimizer->writes, r.rng, 16))
        return POSEIDON_ERR_INVALID_ARG;
    return step(*optimizer, r, stream);
}

extern "C" int poseidon_adamw_values(const poseidon_adamw* optimizer, float* const* m, float* const* v,
                                     hipStream_t stream)
{
    if (!optimizer || (!optimizer->tensors.empty() && (!m || !v)))
        return POSEIDON_ERR_INVALID_ARG;
    try {
        return values(*optimizer, m, v, stream);
    } catch (...) {
        return POSEIDON_ERR_HIP;
    }
}

extern "C" int poseidon_adamw_workspace(const poseidon_adamw* optimizer, int64_t* bytes)
{
    if (!optimizer || !bytes)
        return POSEIDON_ERR_INVALID_ARG;
    *bytes = 8 * optimizer->parts;
    return POSEIDON_OK;
}

extern "C" int poseidon_adamw_clip(const poseidon_adamw* optimizer, double max_norm, float* result, void* workspace,
                                   int64_t workspace_bytes, hipStream_t stream)
{
    if (!optimizer || !(max_norm > 0.0) || !result)
        return POSEIDON_ERR_INVALID_ARG;
    const poseidon_adamw& o = *optimizer;
    const int64_t needed = 8 * o.parts;
    if (needed > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < needed))
        return POSEIDON_ERR_INVALID_ARG;
    if (overlaps(result, 8, workspace, needed) || meets(o.writes, result, 8) || meets(o.reads, result, 8) ||
        meets(o.writes, workspace, needed) || meets(o.reads, workspace, needed))
        return POSEIDON_ERR_INVALID_ARG;
    double* partial = static_cast<double*>(workspace);
    for (int one = 0; one < 2; ++one)
        for (const AdamwGroup& g : o.squares[one]) {
            if (launch_adamw_squares(g, o.dtype, one != 0, partial, stream) != hipSuccess)
                return POSEIDON_ERR_HIP;
            partial += g.blocks;
        }
    return status(launch_adamw_norm(static_cast<const double*>(workspace), o.parts, max_norm, result, stream));
}
