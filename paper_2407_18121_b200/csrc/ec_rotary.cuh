// Arguments of the rotary kernels.
#pragma once

#include "ec_paged.cuh"

namespace ec {

constexpr int kRotaryMostTokens = 16;            // of a CTA

struct RotaryTurn {
    const double *freqs;                         // [rot / 2], radians per position
    int rot;                                     // leading elements of a head that turn; 0: none
    float factor;
    bool inverse;
};

// Strides in 16-byte units.
struct RotaryRows {
    const uint4 *x;
    uint4 *out;
    const int *positions;
    int64_t x_n, x_t, x_h, out_n, out_t, out_h, pos_n;
    int N, T, heads;
};

struct JoinArgs {
    const uint4 *q, *k, *v;                      // packed tokens
    uint4 *q_out;
    const float *w_new;
    const int *slots, *positions;
    int64_t q_t, q_h, qo_t, qo_h, k_t, k_h, v_t, v_h;
    int tokens, Hq;                              // Hq = 0: keys and values alone
};

cudaError_t launch_rotary(const RotaryTurn &r, const RotaryRows &x, int D, int dtype, bool half, cudaStream_t stream);
cudaError_t launch_join(const RotaryTurn &r, const PagedView &c, const JoinArgs &j, int D, int dtype, bool half, cudaStream_t stream);

// Pages of a paged cache handed out and taken back.
struct PagePool {
    int *free, *n_free, *held;
};

struct ReserveArgs {
    const int *counts;
    int *starts, *granted, *slots, *positions;
    int *table, *lens, *seen;
    int tokens, advance, limit;
};

cudaError_t launch_reserve(const PagedView &c, const PagePool &p, const ReserveArgs &a, cudaStream_t stream);
cudaError_t launch_release(const PagedView &c, const PagePool &p, cudaStream_t stream);

}  // namespace ec
