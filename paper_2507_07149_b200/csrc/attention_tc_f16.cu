// float16 instantiation of the tensor-core attention kernels (one translation unit per element type).
#include "attention_tc.cuh"

namespace daf {
template daf_status attn_forward_tc<__half>(const AttnArgs &, WorkspaceHeader *, cudaStream_t);
}
