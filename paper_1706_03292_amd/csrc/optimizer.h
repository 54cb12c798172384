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
    int32_t first_block[ADAMW_GROUP];   // past the last tensor: INT32_MAX
    AdamwItem item[ADAMW_GROUP];
    int64_t chunk;                      // a multiple of ADAMW_CHUNK
    int32_t count;
    int32_t blocks;
};
static_assert(ADAMW_GROUP % 8 == 0, "read eight by eight");
static_assert(sizeof(AdamwGroup) <= 4000, "kernel arguments");

// Values of a workgroup's turn.  A step's workgroup has one turn: with four, VGG19-22K's
// 229M values take 1282 us against 1244 (fp32 moments), 687 against 654 (8 bits).
constexpr int64_t ADAMW_CHUNK = 2048;
constexpr int64_t ADAMW_MOST_BLOCKS = int64_t(1) << 23;   // of a launch: 2^31 threads

// What a launch's tensors have in common for the step: 8-bit moments, one row of
// gradients.
struct AdamwKind {
    bool coded, one;
};

hipError_t launch_adamw_step(const AdamwGroup& group, int32_t dtype, AdamwKind kind, const poseidon_adamw_rule& rule,
                             hipStream_t stream);
hipError_t launch_adamw_values(const AdamwGroup& group, hipStream_t stream);
// Sums of squares, one of each workgroup, to partial[0 .. group.blocks).
// (`one`: one row of gradients each)
hipError_t launch_adamw_squares(const AdamwGroup& group, int32_t dtype, bool one, double* partial, hipStream_t stream);
hipError_t launch_adamw_norm(const double* partial, int64_t parts, double max_norm, float* result,
                             hipStream_t stream);

}  // namespace poseidon
