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
// workgroup its tensor's place (int32).
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
struct Args {
    const Tensor *t;
    const int32_t *of;               // tensor of each workgroup
    int32_t groups;
    double lr;
    uint32_t seed;
    float b1, c1, b2, c2;            // beta and 1 - beta
    float rate, root, eps;           // lr / (1 - beta1^t), (1 - beta2^t)^(-1/2)
    const float *grad_scale;         // device scalar, or null
};

hipError_t launch(const Args &a, bool grad_f32, bool eight, hipStream_t s);

}  // namespace adamw
}  // namespace m3
