// Attention over a cache of 4-bit elements (mx4_attention_impl.h), head_dim 64.
#include "mx4_attention_impl.h"

namespace pa {

pa_status launch_mx4_d64(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int shape, hipStream_t stream)
{
    return launch_mx4_dim<64>(a, merge, dtype, shape, stream);
}

}  // namespace pa
