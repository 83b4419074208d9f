// Host side of the operators of prompts and long conversations: argument validation, launch configuration and the
// extern "C" entry points from mcsd_chunk_attention on (mcsd.h).
#include <cmath>

#include "mcsd_chunk.cuh"
#include "mcsd_evict.cuh"
#include "mcsd_launch.cuh"
#include "mcsd_logprobs.cuh"

namespace mcsd {
namespace {

int check_chunk(const mcsd_chunk_desc *d, const mcsd_kv_cache *cache)
{
    if (!d) return MCSD_ERR_NULL;
    const int rc = check_cache(cache);
    if (rc != MCSD_OK) return rc;
    if (d->reserved != 0 || d->batch < 0 || d->n_heads < 1 || d->max_pages < 0 || d->max_new < 0 || d->n_tokens < 0) return MCSD_ERR_SHAPE;
    if (d->n_heads % cache->n_heads != 0) return MCSD_ERR_SHAPE;
    if (d->n_heads / cache->n_heads > MCSD_MAX_GROUP || d->max_new > 1 << 24 || d->n_tokens > 0x7fffffffLL) return MCSD_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d->max_pages) * cache->page_size > 0x7fffffffLL - 512) return MCSD_ERR_UNSUPPORTED;
    if (d->dtype != MCSD_DTYPE_BF16 && d->dtype != MCSD_DTYPE_F16) return MCSD_ERR_DTYPE;
    if (d->ld_table < d->max_pages || d->q_token_stride < 0 || d->q_head_stride < 0) return MCSD_ERR_STRIDE;
    return MCSD_OK;
}

ChunkParams chunk_params(const mcsd_chunk_desc *d, const mcsd_kv_cache *cache, const int32_t *table, const int32_t *start, const int32_t *cu, const void *q)
{
    ChunkParams p = {};
    p.c = cache_params(cache);
    p.q = q; p.table = table; p.start = start; p.cu = cu;
    p.ld_table = d->ld_table; p.n_tokens = d->n_tokens;
    p.q_token = d->q_token_stride; p.q_head = d->q_head_stride;
    p.o_token = d->out_token_stride; p.o_head = d->out_head_stride;
    p.batch = d->batch; p.n_heads = d->n_heads; p.max_pages = d->max_pages; p.max_new = d->max_new;
    p.group = d->n_heads / cache->n_heads;
    p.scale = d->scale;
    return p;
}

template <int DT, int D>
int launch_chunk(const ChunkParams &p, cudaStream_t st)
{
    const unsigned z = static_cast<unsigned>(p.max_new < 8 ? 1 : p.max_new > 512 ? 64 : p.max_new / 8);
    chunk_kernel<DT, D><<<dim3(p.n_heads, p.batch < 65535 ? p.batch : 65535, z), 256, 0, st>>>(p);
    return launched(1);
}

template <int DT, int D>
int launch_weigh(const ChunkParams &p, cudaStream_t st)
{
    weigh_kernel<DT, D><<<dim3(p.c.n_heads, p.batch < 65535 ? p.batch : 65535, 64), 256, 0, st>>>(p);
    return launched(1);
}

}  // namespace
}  // namespace mcsd

using namespace mcsd;

extern "C" {

size_t mcsd_chunk_attention_workspace_bytes(const mcsd_chunk_desc *desc, const mcsd_kv_cache *cache)
{
    if (check_chunk(desc, cache) != MCSD_OK) return 0;
    return 256;
}

int mcsd_chunk_attention(const mcsd_chunk_desc *desc, const mcsd_kv_cache *cache, const int32_t *page_table, const int32_t *start,
                         const int32_t *cu_tokens, const void *q, void *out, float *lse)
{
    const int rc = check_chunk(desc, cache);
    if (rc != MCSD_OK) return rc;
    const int64_t row = cache->head_dim;
    if ((desc->n_heads > 1 && desc->out_head_stride < row) || (desc->n_tokens > 1 && desc->out_token_stride < row) || desc->out_head_stride < 0 ||
        desc->out_token_stride < 0)
        return MCSD_ERR_STRIDE;
    if (!std::isfinite(desc->scale)) return MCSD_ERR_SHAPE;
    set_last_launches(0);
    if (desc->batch == 0 || desc->n_tokens == 0 || desc->max_new == 0) return MCSD_OK;
    if (!start || !cu_tokens || !q || !out || (!page_table && desc->max_pages > 0)) return MCSD_ERR_NULL;
    if (!on_multiples(2, q, out) || !on_multiples(4, page_table, start, cu_tokens, lse)) return MCSD_ERR_STRIDE;
    if (!desc->workspace || reinterpret_cast<uintptr_t>(desc->workspace) % 256 != 0 ||
        desc->workspace_bytes < mcsd_chunk_attention_workspace_bytes(desc, cache))
        return MCSD_ERR_WORKSPACE;
    ChunkParams p = chunk_params(desc, cache, page_table, start, cu_tokens, q);
    p.out = out;
    p.lse = lse;
    cudaStream_t st = static_cast<cudaStream_t>(desc->stream);
    const bool bf = desc->dtype == MCSD_DTYPE_BF16;
    if (cache->head_dim == 128) return bf ? launch_chunk<MCSD_DTYPE_BF16, 128>(p, st) : launch_chunk<MCSD_DTYPE_F16, 128>(p, st);
    return bf ? launch_chunk<MCSD_DTYPE_BF16, 64>(p, st) : launch_chunk<MCSD_DTYPE_F16, 64>(p, st);
}

int mcsd_accumulate_weights(const mcsd_chunk_desc *desc, const mcsd_kv_cache *cache, const int32_t *page_table, const int32_t *start,
                            const int32_t *cu_tokens, const void *q, const float *lse, float *weights, float decay, int32_t last_tokens)
{
    const int rc = check_chunk(desc, cache);
    if (rc != MCSD_OK) return rc;
    if (!std::isfinite(desc->scale) || !std::isfinite(decay) || last_tokens < 0) return MCSD_ERR_SHAPE;
    set_last_launches(0);
    if (desc->batch == 0 || desc->n_tokens == 0 || desc->max_new == 0 || desc->max_pages == 0 || cache->n_pages == 0) return MCSD_OK;
    if (!start || !cu_tokens || !q || !lse || !weights || !page_table) return MCSD_ERR_NULL;
    if (!on_multiples(2, q) || !on_multiples(4, page_table, start, cu_tokens, lse, weights)) return MCSD_ERR_STRIDE;
    ChunkParams p = chunk_params(desc, cache, page_table, start, cu_tokens, q);
    p.lse = const_cast<float *>(lse);
    p.weights = weights;
    p.decay = decay;
    p.last = last_tokens;
    cudaStream_t st = static_cast<cudaStream_t>(desc->stream);
    const bool bf = desc->dtype == MCSD_DTYPE_BF16;
    if (cache->head_dim == 128) return bf ? launch_weigh<MCSD_DTYPE_BF16, 128>(p, st) : launch_weigh<MCSD_DTYPE_F16, 128>(p, st);
    return bf ? launch_weigh<MCSD_DTYPE_BF16, 64>(p, st) : launch_weigh<MCSD_DTYPE_F16, 64>(p, st);
}

int mcsd_evict_rows(const mcsd_evict_desc *d, const mcsd_kv_cache *cache)
{
    if (!d) return MCSD_ERR_NULL;
    const int rc = check_cache(cache);
    if (rc != MCSD_OK) return rc;
    if (d->reserved != 0 || d->batch < 0 || d->max_pages < 0 || d->keep < 0 || d->sink < 0 || d->recent < 0 || d->n_layers < 1) return MCSD_ERR_SHAPE;
    if (static_cast<int64_t>(d->max_pages) * cache->page_size > 0x7fffffffLL - 512) return MCSD_ERR_UNSUPPORTED;
    if (d->ld_table < d->max_pages || d->layer_stride % 16 != 0 || d->layer_stride < 0 || d->weight_stride < 0) return MCSD_ERR_STRIDE;
    if (d->n_layers > 1 && (d->layer_stride < static_cast<int64_t>(mcsd_kv_block_bytes(cache->head_dim, cache->page_size)) * cache->n_heads ||
                            d->weight_stride < static_cast<int64_t>(cache->n_pages) * cache->n_heads * cache->page_size))
        return MCSD_ERR_STRIDE;
    set_last_launches(0);
    if (d->batch == 0) return MCSD_OK;
    if (!d->len || (!d->page_table && d->max_pages > 0) || (!d->weights && cache->n_pages > 0)) return MCSD_ERR_NULL;
    if (d->len_out == d->len) return MCSD_ERR_SHAPE;
    if (!on_multiples(4, d->page_table, d->len, d->keep_len, d->weights, d->len_out)) return MCSD_ERR_STRIDE;
    if (d->n_layers > (1LL << 40) / (static_cast<int64_t>(d->batch) * cache->n_heads)) return MCSD_ERR_UNSUPPORTED;
    EvictParams p = {};
    p.c = cache_params(cache);
    p.n_layers = d->n_layers; p.layer_stride = d->layer_stride; p.weight_stride = d->weight_stride; p.ld_table = d->ld_table;
    p.table = d->page_table; p.len = d->len; p.keep_len = d->keep_len; p.weights = d->weights; p.len_out = d->len_out;
    p.batch = d->batch; p.max_pages = d->max_pages; p.keep = d->keep; p.sink = d->sink; p.recent = d->recent;
    const long long items = d->n_layers * d->batch * cache->n_heads;
    const unsigned grid = static_cast<unsigned>(items < 1 << 20 ? items : 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(d->stream);
    if (cache->head_dim == 128) evict_kernel<128><<<grid, kEvictThreads, 0, st>>>(p);
    else evict_kernel<64><<<grid, kEvictThreads, 0, st>>>(p);
    return launched(1);
}

int mcsd_token_logprobs(const mcsd_logprob_desc *d)
{
    if (!d) return MCSD_ERR_NULL;
    if (d->reserved != 0 || d->vocab < 1 || d->n_given < 0 || d->n_top < 0 || d->n_logits < 0 || d->n_out < 0) return MCSD_ERR_SHAPE;
    if (d->n_top > d->vocab) return MCSD_ERR_SHAPE;
    if (d->vocab > MCSD_MAX_VOCAB || d->n_top > MCSD_MAX_TOP || d->n_out > 0x7fffffffLL) return MCSD_ERR_UNSUPPORTED;
    if (!good_dtype(d->dtype)) return MCSD_ERR_DTYPE;
    if (!(d->temperature > 0.f) || !std::isfinite(d->temperature) || !std::isfinite(1.f / d->temperature)) return MCSD_ERR_TEMPERATURE;
    if (d->path_nodes && (d->row_index || d->path_len < 1 || d->nodes_per_tree < 1 || d->n_out % d->path_len != 0)) return MCSD_ERR_SHAPE;
    if (d->ld < d->vocab) return MCSD_ERR_STRIDE;
    set_last_launches(0);
    if (d->n_out == 0 || d->n_logits == 0) return MCSD_OK;
    if (!d->logits || (d->logprobs && d->n_given > 0 && !d->tokens)) return MCSD_ERR_NULL;
    if (!on_multiples(static_cast<unsigned>(elem_size(d->dtype)), d->logits) ||
        !on_multiples(4, d->row_index, d->path_nodes, d->tokens, d->logprobs, d->entropy, d->top_ids, d->top_logprobs))
        return MCSD_ERR_STRIDE;
    LogprobParams p = {};
    p.logits = d->logits; p.ld = d->ld; p.n_logits = d->n_logits; p.n_out = d->n_out;
    p.row_index = d->row_index; p.path_nodes = d->path_nodes; p.tokens = d->tokens;
    p.logprobs = d->n_given > 0 ? d->logprobs : nullptr; p.entropy = d->entropy; p.top_ids = d->top_ids; p.top_logprobs = d->top_logprobs;
    p.V = d->vocab; p.n_given = d->n_given; p.n_top = d->top_ids || d->top_logprobs ? d->n_top : 0; p.path_len = d->path_len; p.nodes_per_tree = d->nodes_per_tree;
    p.inv_t = 1.f / d->temperature;
    const unsigned grid = static_cast<unsigned>(d->n_out < 1 << 20 ? d->n_out : 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(d->stream);
    switch (d->dtype) {
    case MCSD_DTYPE_F32: logprob_kernel<MCSD_DTYPE_F32><<<grid, kLogprobThreads, 0, st>>>(p); break;
    case MCSD_DTYPE_BF16: logprob_kernel<MCSD_DTYPE_BF16><<<grid, kLogprobThreads, 0, st>>>(p); break;
    default: logprob_kernel<MCSD_DTYPE_F16><<<grid, kLogprobThreads, 0, st>>>(p); break;
    }
    return launched(1);
}

}  // extern "C"
