// Kernel arguments of the gated linear recurrence (m3_glr.hip), already
// validated by the front end (m3_layers.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace m3 {
namespace glr {

constexpr int kChunk = 128;      // tokens a tile
constexpr int kFwdWaves = 8, kBwdWaves = 8;
constexpr size_t kCtlBytes = 256;

// Channels a lane of the backward takes of the two that the arrays allow: one
// without the gate, where two workgroups then fit a compute unit's registers, two
// with it, where they do not either way.  Over eleven shapes in bf16, 2048 to
// 65536 tokens of a row or many and 256 to 8192 channels, one channel and two took,
// without the gate, 398 us and 457 (65536 of 2048), 114 and 130 (4 x 2048 of 4096),
// 60 and 71 (32768 of 256), but 40 and 36 (8 x 1024 of 1024); with it 694 and 580,
// 185 and 162, but 60 and 75 (32768 of 256): each side is right in nine of them.
inline int bwd_channels(int V, bool gate) { return gate ? V : 1; }

// Strides in elements; the channel stride is 1.  y, the gradients and dy are
// contiguous [B][L][D].  G: channel groups of 64 V, tiles: ceil(L / kChunk).
struct FwdArgs {
    const void *x, *r, *i, *z;
    const float *A, *init;
    void *y;
    float *final_state, *states;     // states [B][tiles][D] or null
    int64_t B, L, D, G, tiles;
    int64_t x_sb, x_st, r_sb, r_st, i_sb, i_st, z_sb, z_st;
    uint64_t *ctl, *inc, *mapA, *mapC;
    uint32_t spin_max;
};
struct BwdArgs {
    const void *x, *r, *i, *z, *dy;
    const float *A, *states, *dfinal;
    void *dx, *dr, *di, *dz;
    float *dA, *dinit;
    int64_t B, L, D, G, tiles;
    int64_t x_sb, x_st, r_sb, r_st, i_sb, i_st, z_sb, z_st;
    uint64_t *ctl, *inc, *mapA, *mapC, *part;
    uint32_t spin_max;
};
struct StepArgs {
    float *state;
    const void *x, *r, *i, *z;
    const float *A;
    void *y;
    int64_t B, D;
    int64_t x_sb, r_sb, i_sb, z_sb;
};

hipError_t launch_fwd(const FwdArgs &a, bool f32, int V, hipStream_t s);
hipError_t launch_bwd(const BwdArgs &a, bool f32, int V, hipStream_t s);
hipError_t launch_step(const StepArgs &a, bool f32, int V, hipStream_t s);

}  // namespace glr
}  // namespace m3
