// What the kernels of the microscaled 4-bit products share.
#pragma once
#include "mx4_common.h"

namespace mbu {

struct Mx4Args {
    const void *x;              // held: codes [M][kp/2]; float: rows `ldx` apart
    const uint8_t *xs;          // held: scales [M][kp/32]
    const void *w;              // held: codes [N][kp/2]; masked: blob
    const uint8_t *ws;          // held: scales [N][kp/32]
    const float *alpha, *bias;  // [N] or NULL
    void *out;
    long long ldx;
    int M, N, K, kp, steps, tiles_n;
};

enum Mx4Weights { W_HELD, W_MASKED };

// Tiled kernel for many rows (mx4_tile.hip); p.x holds codes
int launch_mx4_tile(const char *fn, const Mx4Args &p, bool masked, int dtype, hipStream_t s);

}  // namespace mbu
