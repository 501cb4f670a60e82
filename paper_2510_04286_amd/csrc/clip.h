// Global gradient norm and clipping (clip.hip).
#pragma once
#include "common.h"

namespace slicemoe {

constexpr int kClipThreads = 256;
constexpr int kClipChunks = 8192;   // (662 us for 1.2 GB; 2048: 724, 4096: 671, 16384: 693)
struct ClipPlan {
    int chunk;          // elements per chunk
    long long chunks;   // of all tensors: one 64-bit partial sum each
    bool once;          // whether one block adds them up for all
};
ClipPlan clip_plan(const slicemoe_grad *g, int count);
hipError_t launch_clip_grads(const slicemoe_grad *g, int count, const ClipPlan &plan, float max_norm, float *norm, double *part, hipStream_t s);

}  // namespace slicemoe
