// sk_packed.h -- launchers of the rows in 8 bits, and of the activations that keep them.
#pragma once

#include "sk_routed.h"

namespace sk {

constexpr int kPackBlock = 128;  // columns under one scale, where it is not the whole row

struct PackArgs {
    const void *x, *gy;
    void *y, *gx;
    int8_t *values;
    float *scales;
    int64_t rows;
    int columns, pitch, blocks;  // blocks: scales of a row
    int dtype, kind, gated;
    int gy32;  // gy is in 32 bits, whatever dtype is
    int lanes;
};
inline int pack_pitch(int columns) { return (columns + 15) / 16 * 16; }
hipError_t launch_pack(const PackArgs &a, hipStream_t st);
hipError_t launch_unpack(const PackArgs &a, hipStream_t st);
hipError_t launch_activation_forward(const PackArgs &a, hipStream_t st);
hipError_t launch_activation_backward(const PackArgs &a, hipStream_t st);

}  // namespace sk
