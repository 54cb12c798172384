// What the AdamW kernels' launchers and the optimizer object share.
#pragma once

#include "common.h"

namespace poseidon {

constexpr int ADAMW_BLOCK = 128;   // values that share an exponent byte

// One tensor as the kernels see it (kernel arguments, by value).
struct AdamwItem {
    float* W;            // step; values: where m goes
    const void* G;       // the workers' rows (clip, step)
    void* m;
    void* v;
    uint8_t* exponents;
    void* copy;          // step: bf16 copy; values: where v goes; clip: where the sum goes
    int64_t n;
    int64_t stride;
    int64_t first_group; // the random numbers' group of its first value
    int32_t P;
    float weight_decay;
};

// Tensors of one launch: as many as kernel arguments of 4 KB hold.  Tensor t
// owns the workgroups [first_block[t], first_block[t+1]), `chunk` values each.
constexpr int ADAMW_GROUP = 40;
struct AdamwGroup {
    int32_t first_block[ADAMW_GROUP];
    AdamwItem item[ADAMW_GROUP];
    int32_t count;
    int32_t blocks;
};
static_assert(sizeof(AdamwGroup) <= 4000, "kernel arguments");

// Values that a workgroup of the step (and of values) works on.
constexpr int64_t ADAMW_CHUNK = 2048;
constexpr int64_t ADAMW_MOST_BLOCKS = int64_t(1) << 23;   // of a launch: 2^31 threads

// Kinds of arrays that a group's tensors have.
hipError_t launch_adamw_step(const AdamwGroup& group, int32_t dtype, bool coded, const poseidon_adamw_rule& rule,
                             hipStream_t stream);
hipError_t launch_adamw_values(const AdamwGroup& group, hipStream_t stream);
// Sums of squares, one of each workgroup, to partial[0 .. group.blocks).
hipError_t launch_adamw_squares(const AdamwGroup& group, int32_t dtype, int64_t chunk, double* partial,
                                hipStream_t stream);
hipError_t launch_adamw_norm(const double* partial, int64_t parts, double max_norm, float* result,
                             hipStream_t stream);

}  // namespace poseidon
