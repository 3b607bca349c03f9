// Matrix-core attention of drafted trees (tree_mfma_impl.h) in 256 columns.
#include "tree_mfma_impl.h"

namespace pa {

pa_status launch_tree_d256(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int row_waves, hipStream_t stream)
{
    return launch_tree_dim<256>(a, merge, dtype, row_waves, stream);
}

}  // namespace pa
