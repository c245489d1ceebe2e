// Kernel arguments of the AdamW step (m3_adamw.hip), already validated by the
// front end (m3_layers.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace m3 {
namespace adamw {

constexpr int kBlockElems = 256;     // elements that share the scales of 8-bit states
constexpr int kChunkElems = 1024;    // elements a workgroup

// A table on the device: the tensors that have elements, then for each
// workgroup its tensor's place (int32), then, on 16 bytes, a Now.
struct Tensor {
    float *p;
    const void *g;
    void *m, *v;
    void *low;           // bf16 copy of p, or null
    float *scales;       // [blocks][2], 8-bit states only
    int32_t first, chunks, tail;    // first workgroup, workgroups, elements of the last one
    uint32_t index;      // place in the call's list
    double decay;
};
// What changes from step to step
struct Now {
    double lr;
    float rate, root;                // lr / (1 - beta1^t), (1 - beta2^t)^(-1/2)
    uint32_t seed, unused[3];
};
__host__ __device__ inline Now now(double lr, double beta1, double beta2, int64_t t, uint64_t seed) {
    const double bc1 = 1.0 - pow(beta1, (double)t), bc2 = 1.0 - pow(beta2, (double)t);
    return Now{lr, (float)(lr / bc1), (float)pow(bc2, -0.5), (uint32_t)seed, {}};
}
struct Args {
    const Tensor *t;
    const int32_t *of;               // tensor of each workgroup
    int32_t groups;
    Now now;
    const Now *from;                 // device: read in place of `now`, or null
    float b1, c1, b2, c2, eps;       // beta and 1 - beta
    const float *grad_scale;         // device scalar, or null
};
// A step whose numbers are on the device: what `to` becomes (one thread)
struct NowArgs {
    Now *to;
    double lr, beta1, beta2;
    int64_t step;
    uint64_t seed;
    const int64_t *device_step;      // (null: step)
    const double *device_lr;         // (null: lr)
};

hipError_t launch_now(const NowArgs &a, hipStream_t s);
hipError_t launch(const Args &a, bool grad_f32, bool eight, hipStream_t s);

}  // namespace adamw
}  // namespace m3
