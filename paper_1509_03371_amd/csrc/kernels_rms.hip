// Root-mean-square norm over the channels of a position: which kernels take a call.
#include "rms.h"

namespace sk {

hipError_t launch_rms_norm(const RmsArgs &a, hipStream_t stream)
{
    return a.layout == ROWS ? launch_rms_rows(a, stream) : launch_rms_maps(a, stream);
}

// (one workgroup writes the sums itself)
size_t rms_bwd_scratch_floats(const NormSpan &s)
{
    if (s.n * s.plane == 0) return 0;
    const int copies = s.layout == ROWS ? rms_rows_bwd_copies(s) : rms_maps_bwd_copies(s);
    return copies > 1 ? (size_t)copies * rms_copy_floats(s.c) : 0;
}

hipError_t launch_rms_norm_bwd(const RmsBwdArgs &a, hipStream_t stream)
{
    if (a.n * a.plane == 0) return a.dgamma ? launch_rms_reduce(nullptr, 0, a.dgamma, a.c, stream) : hipSuccess;
    return a.layout == ROWS ? launch_rms_rows_bwd(a, stream) : launch_rms_maps_bwd(a, stream);
}

}  // namespace sk
