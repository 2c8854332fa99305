// Layer norm over the channels of a position: which kernels take a call.
#include "norm_device.h"

namespace sk {

hipError_t launch_layer_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.n * a.plane == 0) return hipSuccess;
    return a.layout == ROWS ? launch_norm_rows(a, stream) : launch_norm_planes(a, stream);
}

static int wanted_copies(const NormSpan &s)
{
    if (s.n * s.plane == 0) return 0;
    return s.layout == ROWS ? norm_rows_bwd_copies(s) : norm_planes_bwd_copies(s);
}

// (one workgroup writes the sums themselves)
size_t norm_bwd_scratch_floats(const NormSpan &s)
{
    const int copies = wanted_copies(s);
    return copies > 1 ? (size_t)copies * norm_copy_floats(s.c) : 0;
}

hipError_t launch_layer_norm_bwd(const NormBwdArgs &a, hipStream_t stream)
{
    const bool sums = a.dgamma || a.dbeta;
    int copies = wanted_copies(a);
    if (copies == 0) return sums ? launch_norm_reduce(nullptr, 0, a.dgamma, a.dbeta, a.c, stream) : hipSuccess;
    if (sums) copies = (int)std::max<size_t>(1, std::min<size_t>(copies, a.scratch_floats / norm_copy_floats(a.c)));
    return a.layout == ROWS ? launch_norm_rows_bwd(a, copies, stream) : launch_norm_planes_bwd(a, copies, stream);
}

}  // namespace sk
