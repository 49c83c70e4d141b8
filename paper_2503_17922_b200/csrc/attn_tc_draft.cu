// Attention on the tensor cores: drafted tokens over a cache of plain rows.
#include "attn_tc_kernel.cuh"

namespace wkv {

cudaError_t launch_tc_draft(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    return launch_tc_form<false, true>(t, k_map, v_map, stream);
}

}  // namespace wkv
