// Activations in 8 bits, root-mean-square norm: launchers (internal to libsknet).
#pragma once
#include "norm.h"

namespace sk {

enum { E4M3 = 0, I8 = 1 };

// One operand in 8 bits: codes as a NormView of bytes; scales of a line at b*ssn (+ channel*ssc for MAPS), one byte a block of 32.
struct PackedView {
    uint8_t *codes = nullptr, *scales = nullptr;
    long sn = 0, sc = 0, ssn = 0, ssc = 0;
    int code = E4M3;
};

struct Pack8Args : NormSpan {
    NormView x;                  // unpacking: the result
    PackedView packed;
};
hipError_t launch_pack8(const Pack8Args &a, hipStream_t stream);
hipError_t launch_unpack8(const Pack8Args &a, hipStream_t stream);

// s = x + residual; y = s rstd gamma
struct RmsArgs : NormSpan {
    NormView x, residual, sum, y;      // residual, sum, y optional
    PackedView sum8, y8;               // optional
    const float *gamma;                // optional
    float *rstd;                       // optional
    float eps;
};
hipError_t launch_rms_norm(const RmsArgs &a, hipStream_t stream);

// dx = rstd (g - h mean_c(g h)) + dsum with h = s rstd, g = gamma dy
struct RmsBwdArgs : NormSpan {
    NormView dy, s, dsum, dx;          // s or s8; dsum, dx optional
    PackedView s8;
    const float *rstd, *gamma;         // gamma optional
    float *dgamma;                     // optional, [c]
    float *scratch;                    // rms_bwd_scratch_floats of them, if dgamma is asked for
};
size_t rms_bwd_scratch_floats(const NormSpan &s);
hipError_t launch_rms_norm_bwd(const RmsBwdArgs &a, hipStream_t stream);

// dw[o][k] (+)= sum over positions of dy[q][o] x[q][k]; db[o] (+)= sum of dy[q][o]
struct Wgrad8Args : NormSpan {         // dtype: dy's
    long c_out;
    NormView dy;
    PackedView x;
    int accumulate;
    float *dw, *db;                    // db optional
    float *scratch;                    // wgrad8_scratch_floats of them
};
size_t wgrad8_scratch_floats(const NormSpan &s, long c_out);
hipError_t launch_wgrad8(const Wgrad8Args &a, hipStream_t stream);

}  // namespace sk
