// Launchers of layer norm and dropout (internal to libsknet).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "philox.h"

namespace sk {

// How the channels of a position lie: side by side (ROWS, plane = 1), one map after the other (MAPS), or in octets
// [n][ceil(c/8)][plane][8] as the 16-bit nets keep them (OCTETS; written whole, zeros behind the last channel).
enum { ROWS = 0, MAPS = 1, OCTETS = 2 };

// One operand.  In elements of its type: ROWS b*sn + c; MAPS b*sn + c*sc + m; OCTETS b*sn + (c/8)*sc + 8*m + c%8.
struct NormView {
    void *p = nullptr;
    long sn = 0, sc = 0;
};

struct NormSpan {
    int dtype, layout;           // SK_F32 / SK_BF16 / SK_F16
    long n, plane;
    int c;
};

struct DropoutArgs : NormSpan {
    NormView x, y;
    NormView relu_src;           // optional: y = 0 where this is not > 0 (the ReLU in front of the layer, backwards)
    DropMask drop;
};
hipError_t launch_dropout(const DropoutArgs &a, hipStream_t stream);

// s = residual + dropout(x); y = (s - mean) rstd gamma + beta, then max(0, .) if relu
struct NormArgs : NormSpan {
    NormView x, residual, sum, y;     // residual, sum optional
    const float *gamma, *beta;        // optional
    float *mean, *rstd;               // optional, [n][plane]
    float eps;
    int relu;
    DropMask drop;
};
hipError_t launch_layer_norm(const NormArgs &a, hipStream_t stream);

// t = rstd (g - mean_c(g) - h mean_c(g h)) + dsum with h = (s - mean) rstd, g = gamma dy; dresidual = t; dx = dropout(t), 0 where relu_x and s <= 0
struct NormBwdArgs : NormSpan {
    NormView dy, s, dsum, dx, dresidual;   // dsum, dx, dresidual optional
    const float *mean, *rstd, *gamma;      // gamma optional
    float *dgamma, *dbeta;                 // optional, [c]
    float *scratch;                        // partial sums of dgamma and dbeta
    size_t scratch_floats;
    int relu_x;
    DropMask drop;
    // does a result go to the place of what the parameters' sums are made from?
    bool in_place() const
    {
        for (const void *out : {dx.p, dresidual.p})
            if (out && (out == dy.p || out == s.p)) return true;
        return false;
    }
};
size_t norm_bwd_scratch_floats(const NormSpan &s);        // of the fastest launch; with less, fewer workgroups share the sums out
hipError_t launch_layer_norm_bwd(const NormBwdArgs &a, hipStream_t stream);

// step[0] += 1, one more forward pass, and step[1] = that one's number (a kernel, so that a recorded pass moves on at every replay)
hipError_t launch_step_add(uint64_t *step, hipStream_t stream);

}  // namespace sk
