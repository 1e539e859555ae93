// Entry points of attention: argument checks and the choice of the kernels.
#include "attention.cuh"

namespace daf {

constexpr uint32_t kAttnRowPad = 128;            // rows of the backward workspace are padded to whole tiles

static bool tensor_ok(const void *p, const uint64_t (&st)[3], uint32_t B, uint32_t S, uint32_t H, uint32_t D, uint32_t bytes)
{
    if (!p || (reinterpret_cast<uintptr_t>(p) & 15u)) return false;
    const uint32_t unit = 16u / bytes;           // a row starts on a 16-byte boundary
    const uint32_t extent[3] = {B, S, H};
    for (int i = 0; i < 3; i++)
        // an extent of one has no stride; otherwise elements of two rows must not share memory
        if (extent[i] > 1u && (st[i] < D || st[i] % unit || st[i] >= (1ull << 36))) return false;
    return true;
}

static daf_status check_attention(const daf_attention_params *p)
{
    if (!p || p->struct_size != sizeof(daf_attention_params) || p->dtype > DAF_BF16 || p->reserved[0] || p->reserved[1]) return DAF_ERR_INVALID_ARG;
    if (p->causal > 1u || !(p->scale > -INFINITY && p->scale < INFINITY)) return DAF_ERR_INVALID_ARG;
    if (p->heads == 0 || p->kv_heads == 0 || p->heads % p->kv_heads || p->head_dim == 0 || p->head_dim % 8u) return DAF_ERR_SHAPE;
    if (p->head_dim > 128u || p->queries > (1u << 24) || p->keys > (1u << 24)) return DAF_ERR_UNSUPPORTED;
    const uint64_t heads = (uint64_t)p->batch * p->heads, kv_heads = (uint64_t)p->batch * p->kv_heads;
    if (heads > 65535u || heads * p->queries > (1ull << 32) || kv_heads * p->keys > (1ull << 32)) return DAF_ERR_UNSUPPORTED;
    return DAF_OK;
}

static AttnTensor tensor_of(const void *p, const uint64_t (&st)[3])
{
    return {const_cast<void *>(p), st[0], st[1], st[2]};
}

static bool encode_map(CUtensorMap *map, bool bf16, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D, uint32_t rows, uint32_t elems,
                       CUtensorMapSwizzle swizzle)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<Encode>(fn) : nullptr;
    }();
    if (!encode) return false;
    const cuuint64_t extent[4] = {D, H, S, B}, none = (2ull * D + 15u) & ~15ull;     // an extent of one has no stride of its own
    const cuuint64_t stride[3] = {H > 1u ? 2ull * t.sh : none, S > 1u ? 2ull * t.ss : none, B > 1u ? 2ull * t.sb : none};
    const cuuint32_t box[4] = {elems, 1, rows, 1}, step[4] = {1, 1, 1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, t.p, extent, stride, box, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool attn_tensor_map(CUtensorMap *map, bool bf16, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D, uint32_t rows)
{
    return encode_map(map, bf16, t, B, S, H, D, rows, 64, CU_TENSOR_MAP_SWIZZLE_128B);
}
bool attn_store_map(CUtensorMap *map, bool bf16, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D)
{
    return encode_map(map, bf16, t, B, S, H, D, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
}

static uint32_t padded_rows(uint32_t rows) { return (rows + kAttnRowPad - 1u) / kAttnRowPad * kAttnRowPad; }

uint32_t attn_splits(const AttnArgs &a)
{
    constexpr uint32_t kSms = 148, kTileRows = 256, kKeys = 128, kMinBlocks = 8;
    const uint64_t tiles = (uint64_t)((a.Sq + kTileRows - 1u) / kTileRows) * a.B * a.H, blocks = (a.Sk + kKeys - 1u) / kKeys;
    if (tiles == 0 || 2u * tiles > kSms || blocks < kMinBlocks) return 1;
    const uint64_t room = kSms / tiles, most = blocks / 2u;         // two blocks at least to a split
    return (uint32_t)(room < most ? room : most);
}

// -lse and -delta of every row, for float16 the squared norm of its grad_out, too
static uint64_t rows_bytes(const daf_attention_params *p)
{
    return (p->dtype == DAF_F16 ? 3ull : 2ull) * p->batch * p->heads * padded_rows(p->queries) * sizeof(float);
}
static uint64_t maxima_bytes(const daf_attention_params *p)
{
    return p->dtype == DAF_F16 ? (2ull * p->batch * p->kv_heads * sizeof(float) + 255u) & ~255ull : 0u;
}

// A call with nothing to do: its workspace, which may be missing, says so.
static daf_status no_work(void *d_workspace, uint64_t workspace_bytes, daf_stream stream)
{
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 15u) || workspace_bytes < sizeof(uint32_t)) return DAF_OK;
    return cudaMemsetAsync(d_workspace, 0, sizeof(uint32_t), reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

static AttnArgs args_of(const daf_attention_params *p)
{
    AttnArgs a = {};
    a.B = p->batch;
    a.Sq = p->queries;
    a.Sk = p->keys;
    a.H = p->heads;
    a.Hkv = p->kv_heads;
    a.D = p->head_dim;
    a.group = p->heads / p->kv_heads;
    a.causal = p->causal;
    a.rows_padded = padded_rows(p->queries);
    a.scale = p->scale;
    a.scale_log2 = p->scale * 1.4426950408889634f;
    return a;
}

}  // namespace daf

using namespace daf;

extern "C" uint64_t daf_attention_workspace(const daf_attention_params *params)
{
    if (check_attention(params) != DAF_OK) return 0;
    const AttnArgs a = args_of(params);
    if (params->dtype == DAF_F32) return sizeof(WorkspaceHeader) + attn_planes_workspace(a, false);
    const uint64_t splits = attn_splits(a);
    return sizeof(WorkspaceHeader) + (splits > 1u ? splits * a.B * a.H * a.Sq * (a.D + 1u) * sizeof(float) : 0u);
}

extern "C" daf_status daf_attention(const daf_attention_params *params, const void *d_q, const void *d_k, const void *d_v,
                                    const int32_t *d_key_lengths, void *d_out, float *d_lse, void *d_workspace,
                                    uint64_t workspace_bytes, daf_stream stream)
{
    const daf_status st = check_attention(params);
    if (st != DAF_OK) return st;
    const daf_attention_params &p = *params;
    const uint32_t eb = p.dtype == DAF_F32 ? 4u : 2u;
    if (reinterpret_cast<uintptr_t>(d_key_lengths) & 3u) return DAF_ERR_INVALID_ARG;
    if (p.batch == 0 || p.queries == 0) return no_work(d_workspace, workspace_bytes, stream);
    if (!tensor_ok(d_q, p.q_stride, p.batch, p.queries, p.heads, p.head_dim, eb) || !d_lse || (reinterpret_cast<uintptr_t>(d_lse) & 3u) ||
        !tensor_ok(d_out, p.out_stride, p.batch, p.queries, p.heads, p.head_dim, eb) ||
        (p.keys && (!tensor_ok(d_k, p.k_stride, p.batch, p.keys, p.kv_heads, p.head_dim, eb) ||
                    !tensor_ok(d_v, p.v_stride, p.batch, p.keys, p.kv_heads, p.head_dim, eb))))
        return DAF_ERR_INVALID_ARG;
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 15u)) return DAF_ERR_INVALID_ARG;
    if (workspace_bytes < daf_attention_workspace(params)) return DAF_ERR_CAPACITY;
    AttnArgs a = args_of(params);
    a.q = tensor_of(d_q, p.q_stride);
    a.k = tensor_of(d_k, p.k_stride);
    a.v = tensor_of(d_v, p.v_stride);
    a.out = tensor_of(d_out, p.out_stride);
    a.lse = d_lse;
    a.lengths = d_key_lengths;
    if (!(a.device_status = device_status_word())) return DAF_ERR_CUDA;
    WorkspaceHeader *const header = reinterpret_cast<WorkspaceHeader *>(d_workspace);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return p.dtype == DAF_F32 ? attn_forward_planes(a, reinterpret_cast<char *>(d_workspace) + sizeof(WorkspaceHeader), header, s)
           : p.dtype == DAF_F16 ? attn_forward_tc<__half>(a, header, s) : attn_forward_tc<__nv_bfloat16>(a, header, s);
}

extern "C" uint64_t daf_attention_grad_workspace(const daf_attention_params *params)
{
    if (check_attention(params) != DAF_OK) return 0;
    return sizeof(WorkspaceHeader) + rows_bytes(params) + maxima_bytes(params) + (params->dtype == DAF_F32 ? attn_planes_workspace(args_of(params), true) : 0u);
}

extern "C" daf_status daf_attention_grad(const daf_attention_params *params, const void *d_q, const void *d_k, const void *d_v,
                                         const int32_t *d_key_lengths, const void *d_out, const float *d_lse,
                                         const void *d_grad_out, void *d_grad_q, void *d_grad_k, void *d_grad_v,
                                         void *d_workspace, uint64_t workspace_bytes, daf_stream stream)
{
    const daf_status st = check_attention(params);
    if (st != DAF_OK) return st;
    const daf_attention_params &p = *params;
    const uint32_t eb = p.dtype == DAF_F32 ? 4u : 2u;
    if (reinterpret_cast<uintptr_t>(d_key_lengths) & 3u) return DAF_ERR_INVALID_ARG;
    if (p.batch == 0 || (p.queries == 0 && p.keys == 0)) return no_work(d_workspace, workspace_bytes, stream);
    if (p.queries && (!tensor_ok(d_q, p.q_stride, p.batch, p.queries, p.heads, p.head_dim, eb) || !d_lse || (reinterpret_cast<uintptr_t>(d_lse) & 3u) ||
                      !tensor_ok(d_out, p.out_stride, p.batch, p.queries, p.heads, p.head_dim, eb) ||
                      !tensor_ok(d_grad_out, p.grad_out_stride, p.batch, p.queries, p.heads, p.head_dim, eb) ||
                      !tensor_ok(d_grad_q, p.grad_q_stride, p.batch, p.queries, p.heads, p.head_dim, eb)))
        return DAF_ERR_INVALID_ARG;
    if (p.keys && (!tensor_ok(d_k, p.k_stride, p.batch, p.keys, p.kv_heads, p.head_dim, eb) ||
                   !tensor_ok(d_v, p.v_stride, p.batch, p.keys, p.kv_heads, p.head_dim, eb) ||
                   !tensor_ok(d_grad_k, p.grad_k_stride, p.batch, p.keys, p.kv_heads, p.head_dim, eb) ||
                   !tensor_ok(d_grad_v, p.grad_v_stride, p.batch, p.keys, p.kv_heads, p.head_dim, eb)))
        return DAF_ERR_INVALID_ARG;
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 15u)) return DAF_ERR_INVALID_ARG;
    if (workspace_bytes < daf_attention_grad_workspace(params)) return DAF_ERR_CAPACITY;
    AttnArgs a = args_of(params);
    a.q = tensor_of(d_q, p.q_stride);
    a.k = tensor_of(d_k, p.k_stride);
    a.v = tensor_of(d_v, p.v_stride);
    a.out = tensor_of(d_out, p.out_stride);
    a.grad_out = tensor_of(d_grad_out, p.grad_out_stride);
    a.dq = tensor_of(d_grad_q, p.grad_q_stride);
    a.dk = tensor_of(d_grad_k, p.grad_k_stride);
    a.dv = tensor_of(d_grad_v, p.grad_v_stride);
    a.lse = const_cast<float *>(d_lse);
    a.lengths = d_key_lengths;
    if (!(a.device_status = device_status_word())) return DAF_ERR_CUDA;
    a.row_nl2 = reinterpret_cast<float *>(reinterpret_cast<char *>(d_workspace) + sizeof(WorkspaceHeader));
    a.row_ndelta = a.row_nl2 + (uint64_t)a.B * a.H * a.rows_padded;
    WorkspaceHeader *const header = reinterpret_cast<WorkspaceHeader *>(d_workspace);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    a.row_norm2 = a.row_ndelta + (uint64_t)a.B * a.H * a.rows_padded;
    a.grad_max = a.row_norm2 + (uint64_t)a.B * a.H * a.rows_padded;
    a.value_max = a.grad_max + (uint64_t)a.B * a.Hkv;
    if (maxima_bytes(params) && cudaMemsetAsync(a.grad_max, 0, maxima_bytes(params), s) != cudaSuccess) return DAF_ERR_CUDA;
    if (p.queries) {
        const daf_status rows = attn_rows(p.dtype, a, header, s);
        if (rows != DAF_OK) return rows;
    } else if (cudaMemsetAsync(header, 0, sizeof(uint32_t), s) != cudaSuccess) {
        return DAF_ERR_CUDA;
    }
    if (p.queries == 0) {
        const daf_status st = attn_zero(p.dtype, a.dk, a.B, a.Sk, a.Hkv, a.D, s);
        return st != DAF_OK ? st : attn_zero(p.dtype, a.dv, a.B, a.Sk, a.Hkv, a.D, s);
    }
    if (p.keys == 0) return attn_zero(p.dtype, a.dq, a.B, a.Sq, a.H, a.D, s);
    char *const planes = reinterpret_cast<char *>(d_workspace) + sizeof(WorkspaceHeader) + rows_bytes(params);
    return p.dtype == DAF_F32 ? attn_backward_planes(a, planes, header, s)
           : p.dtype == DAF_F16 ? attn_backward_tc<__half>(a, header, s) : attn_backward_tc<__nv_bfloat16>(a, header, s);
}
