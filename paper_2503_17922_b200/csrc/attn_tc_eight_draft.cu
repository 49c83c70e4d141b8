// Attention on the tensor cores: drafted tokens over the 8-bit cache.
#include "attn_tc_kernel.cuh"

namespace wkv {

cudaError_t launch_tc_eight_draft(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    return launch_tc_form<true, true>(t, k_map, v_map, stream);
}

}  // namespace wkv
