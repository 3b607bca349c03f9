// Attention over a cache of 4-bit elements (mx4_attention_impl.h), head_dim 256.
#include "mx4_attention_impl.h"

namespace pa {

pa_status launch_mx4_d256(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int shape, hipStream_t stream)
{
    return launch_mx4_dim<256>(a, merge, dtype, shape, stream);
}

}  // namespace pa
