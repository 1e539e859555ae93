// bfloat16 instantiation of the tensor-core attention kernels (one translation unit per element type).
#include "attention_tc.cuh"
#include "attention_tc_grad.cuh"

namespace daf {
template daf_status attn_forward_tc<__nv_bfloat16>(const AttnArgs &, WorkspaceHeader *, cudaStream_t);
template daf_status attn_backward_tc<__nv_bfloat16>(const AttnArgs &, WorkspaceHeader *, cudaStream_t);
}
