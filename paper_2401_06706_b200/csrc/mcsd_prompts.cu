// Host side of the operators of prompts and long conversations: argument validation, launch configuration and the
// extern "C" entry points from mcsd_chunk_attention on (mcsd.h).
#include <cmath>
#include <initializer_list>

#include "mcsd_chunk.cuh"
#include "mcsd_chunk_wide.cuh"
#include "mcsd_evict.cuh"
#include "mcsd_launch.cuh"
#include "mcsd_logprobs.cuh"
#include "mcsd_weigh.cuh"

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
    // (rows of a sequence, and those that a last block has room for beyond them, are counted in 32 bits)
    const int64_t most = d->max_new < d->n_tokens ? d->max_new : d->n_tokens;
    if (most * (d->n_heads / cache->n_heads) > 0x7fffffffLL - kChunkRows) return MCSD_ERR_UNSUPPORTED;
    // (the cuts count places of all blocks, and of all units with their rows, in 64 bits)
    const double room = static_cast<double>(d->max_pages) * cache->page_size + d->max_new + 1024.0;
    if ((static_cast<double>(d->n_tokens) + d->batch) * cache->n_heads * room > 4e18) return MCSD_ERR_UNSUPPORTED;
    if (static_cast<double>(d->batch) * d->n_heads * room * (static_cast<double>(d->max_new) + 64.0) > 4e18) return MCSD_ERR_UNSUPPORTED;
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
    p.scale_part = scale_part(d->scale, &p.scale_power);
    p.q_vec = (reinterpret_cast<uintptr_t>(q) | 2ull * static_cast<unsigned long long>(d->q_token_stride | d->q_head_stride)) % 16 == 0;
    return p;
}

void wait_limits(ChunkParams &p)
{
    const int polls = mcsd_get_option(MCSD_OPT_WAIT_POLLS);
    p.wait_polls = polls > 0 ? static_cast<uint32_t>(polls) : kWaitPolls;
    p.test_extra = mcsd_get_option(MCSD_OPT_TEST_EXTRA_TX) > 0 ? 1u : 0u;
}

// Whether many sequences can have far fewer tokens than the longest chunk: those get the kernel for few rows beside the one for many. A
// batch of 24 with three chunks of 253 tokens and 21 of one takes 95 us with both and 131 with the wide one alone. Where all have as many
// tokens, the second launch is for nothing: 57 instead of 50 us (4 chunks of 16 tokens), 29 instead of 26 (weights, 8 windows of 32).
bool mixed(const mcsd_chunk_desc *d) { return d->n_tokens < static_cast<int64_t>(d->batch) * d->max_new / 2; }

// How a call is laid out; depends on the sizes only. Few rows go to the narrow kernel (blocks of up to 24, which decode the keys once for each
// block), others to the wide one (blocks of 256, most of them empty then). 8 key heads of 128 numbers, 4000 keys, 64 sequences and 4, narrow
// against wide in us: 32 rows 183 | 299 and 32 | 47, 64 rows 263 | 319 and 40 | 50, 96 rows 361 | 316 and 48 | 50. So up to three blocks of 24.
constexpr int kChunkNarrowRows = 72;
struct ChunkPlan {
    int narrow;     // rows of the narrow kernel's blocks, 0: it is not needed
    bool wide;
    int most;       // rows of a sequence up to which it is the narrow kernel's (of a call that has both)
    int ctas[2];    // CTAs the work of the narrow and of the wide kernel is cut for
};
ChunkPlan chunk_plan(const mcsd_chunk_desc *d, const mcsd_kv_cache *cache, bool may_mix)
{
    ChunkPlan plan = {};
    int sms = sm_count();
    if (sms <= 0) sms = 148;
    const int group = d->n_heads / cache->n_heads;
    const long long rows = static_cast<long long>(d->max_new) * group;
    // beside the wide kernel the narrow one has the sequences of one token
    const int narrow = group <= 8 ? 8 : group <= 16 ? 16 : group <= 24 ? 24 : 0;
    if (rows <= kChunkNarrowRows && narrow) {
        plan.narrow = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 24 ? 24 : rows <= 32 && group <= 16 ? 16 : 24;
        plan.most = kChunkNarrowRows;
    } else {
        plan.wide = true;
        if (may_mix && narrow) {
            plan.narrow = narrow;
            plan.most = narrow;
        }
    }
    plan.ctas[0] = plan.narrow ? sms * (plan.narrow == 8 ? kNarrowCtas<1> : plan.narrow == 16 ? kNarrowCtas<2> : kNarrowCtas<3>) : 0;
    plan.ctas[1] = plan.wide ? sms : 0;
    return plan;
}

// Bytes of the notes on divided blocks, ahead of the partial results in the workspace.
size_t join_bytes(const ChunkPlan &plan) { return (sizeof(ChunkJoin) * static_cast<size_t>(plan.ctas[0] > plan.ctas[1] ? plan.ctas[0] : plan.ctas[1]) + 255) / 256 * 256; }

// Launches the kernel that does the work and, as its programmatic dependent, the one that joins divided blocks.
template <int DT, int D, int ROWS, auto Kernel>
int launch_with_join(int threads, int smem, const ChunkParams &p, cudaStream_t st)
{
    if (!allow_smem<Kernel>(smem)) return MCSD_ERR_CUDA;
    Kernel<<<p.n_ctas, threads, smem, st>>>(p);
    if (cudaGetLastError() != cudaSuccess) return MCSD_ERR_CUDA;
    if (p.n_ctas < 2) return MCSD_OK;
    cudaLaunchConfig_t cfg = {};
    constexpr int kRows = kChunkJoinThreads / (D / 4);
    cfg.gridDim = dim3(static_cast<unsigned>(p.n_ctas - 1), (ROWS + kRows - 1) / kRows);
    cfg.blockDim = dim3(kChunkJoinThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, chunk_join_kernel<DT, D, ROWS>, p) == cudaSuccess ? MCSD_OK : MCSD_ERR_CUDA;
}

// Places of the cut that a block costs beside its keys: its queries, its results and the first unit's way through the kernel. Six prompts of 80 to
// 2041 tokens 435 us at 256, 416 at 512, 431 at 1024; 64 sequences of 6 tokens (narrow kernel) 116, 111 and 116.
constexpr int kChunkLead = 512;

template <int DT, int D>
int launch_chunk(ChunkParams p, const ChunkPlan &plan, cudaStream_t st)
{
    int rc = MCSD_OK;
    if (plan.wide) {
        p.tokens = kChunkRows / p.group;
        p.least = plan.narrow ? plan.most + 1 : 0;
        p.most = 0x7fffffff;
        p.lead = kChunkLead;
        p.n_ctas = plan.ctas[1];
        rc = launch_with_join<DT, D, kChunkRows, chunk_wide_kernel<DT, D>>(kChunkThreads, kChunkSmem<D>, p, st);
    }
    if (plan.narrow && rc == MCSD_OK) {
        p.tokens = plan.narrow / p.group;
        p.least = 0;
        p.most = plan.wide ? plan.most : 0x7fffffff;
        p.lead = kChunkLead;
        p.n_ctas = plan.ctas[0];
        if (plan.narrow == 8) rc = launch_with_join<DT, D, 8, narrow_kernel<DT, D, 1, ChunkRows>>(kNarrowWarps * 32, kNarrowSmem<D, 1>, p, st);
        else if (plan.narrow == 16) rc = launch_with_join<DT, D, 16, narrow_kernel<DT, D, 2, ChunkRows>>(kNarrowWarps * 32, kNarrowSmem<D, 2>, p, st);
        else rc = launch_with_join<DT, D, 24, narrow_kernel<DT, D, 3, ChunkRows>>(kNarrowWarps * 32, kNarrowSmem<D, 3>, p, st);
    }
    return rc == MCSD_OK ? launched(plan.wide && plan.narrow ? 4 : 2) : rc;
}

// Places that a (sequence, key head) costs beside its units. Hardly felt: decoding batch 25.4, 25.2 and 27.3 us at 32, 128 and 384, windows of 32 tokens
// (wide kernel) 27.1, 25.7 and 25.3 at 64, 256 and 1024.
constexpr int kWeighLeadNarrow = 128, kWeighLeadWide = 256;

template <int DT, int D, int NB>
int launch_weigh_narrow(ChunkParams p, int sms, cudaStream_t st)
{
    if (!allow_smem<weigh_narrow_kernel<DT, D, NB>>(kWeighSmem<D>)) return MCSD_ERR_CUDA;
    p.lead = kWeighLeadNarrow;
    p.n_ctas = sms * kWeighCtas<NB>;
    weigh_narrow_kernel<DT, D, NB><<<p.n_ctas, kNarrowWarps * 32, kWeighSmem<D>, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? MCSD_OK : MCSD_ERR_CUDA;
}

// Sequences of few rows (their tokens that count x query heads of a key head: what one block of the narrow kernel holds) go to the narrow kernel,
// others to the wide one; a call with rows for the wide one launches both only where there can be many sequences of the other kind. 32 sequences of
// 4000 keys, 8 key heads, narrow against wide: 25 | 46 us with 4 rows, 28 | 48 with 16, 34 | 48 with 24.
template <int DT, int D>
int launch_weigh(ChunkParams p, bool may_mix, cudaStream_t st)
{
    const int sms = sm_count();
    if (sms <= 0) return MCSD_ERR_CUDA;
    const long long rows = static_cast<long long>(p.last > 0 && p.last < p.max_new ? p.last : p.max_new) * p.group;
    const int narrow = rows <= 24 ? static_cast<int>(rows) : may_mix && p.group <= 24 ? p.group : 0;
    int rc = MCSD_OK, n = 0;
    if (rows > 24) {
        if (!allow_smem<weigh_wide_kernel<DT, D>>(kWeighWideSmem<D>)) return MCSD_ERR_CUDA;
        p.least = narrow ? narrow + 1 : 0;
        p.most = 0x7fffffff;
        p.lead = kWeighLeadWide;
        p.n_ctas = sms;
        weigh_wide_kernel<DT, D><<<p.n_ctas, kWeighThreads, kWeighWideSmem<D>, st>>>(p);
        if (cudaGetLastError() != cudaSuccess) return MCSD_ERR_CUDA;
        ++n;
    }
    if (narrow) {
        p.least = 0;
        p.most = rows > 24 ? narrow : 0x7fffffff;
        rc = narrow <= 8 ? launch_weigh_narrow<DT, D, 1>(p, sms, st) : narrow <= 16 ? launch_weigh_narrow<DT, D, 2>(p, sms, st) : launch_weigh_narrow<DT, D, 3>(p, sms, st);
        ++n;
    }
    return rc == MCSD_OK ? launched(n) : rc;
}

// Rows that leave multiprocessors idle get CTAs of 1024 threads (their latency counts), others 256, eight to a multiprocessor: rows of 32000 bf16
// logits and 20 tokens 13 | 17 us at 100 rows, 21 | 19 at 200, 67 | 31 at 1000.
template <int DT>
int launch_logprobs(const LogprobParams &p, bool vec, cudaStream_t st)
{
    const long long sms = sm_count();
    if (sms <= 0) return MCSD_ERR_CUDA;
    const bool few = p.n_out <= sms;
    const unsigned grid = static_cast<unsigned>(p.n_out);
    if (few) {
        if (vec) logprob_kernel<DT, 1024, true><<<grid, 1024, 0, st>>>(p);
        else logprob_kernel<DT, 1024, false><<<grid, 1024, 0, st>>>(p);
    } else {
        if (vec) logprob_kernel<DT, 256, true><<<grid, 256, 0, st>>>(p);
        else logprob_kernel<DT, 256, false><<<grid, 256, 0, st>>>(p);
    }
    return launched(1);
}

}  // namespace
}  // namespace mcsd

using namespace mcsd;

extern "C" {

size_t mcsd_chunk_attention_workspace_bytes(const mcsd_chunk_desc *desc, const mcsd_kv_cache *cache)
{
    if (check_chunk(desc, cache) != MCSD_OK) return 0;
    const ChunkPlan plan = chunk_plan(desc, cache, true);
    const size_t narrow = static_cast<size_t>(plan.ctas[0]) * part_floats(plan.narrow, cache->head_dim);
    const size_t wide = static_cast<size_t>(plan.ctas[1]) * part_floats(kChunkRows, cache->head_dim);
    return join_bytes(plan) + (2 * sizeof(float) * (narrow > wide ? narrow : wide) + 255) / 256 * 256;
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
    p.o_vec = (reinterpret_cast<uintptr_t>(out) | 2ull * static_cast<unsigned long long>(desc->out_token_stride | desc->out_head_stride)) % 16 == 0;
    wait_limits(p);
    const ChunkPlan plan = chunk_plan(desc, cache, mixed(desc));
    p.joins = static_cast<ChunkJoin *>(desc->workspace);
    p.part = reinterpret_cast<float *>(static_cast<char *>(desc->workspace) + join_bytes(chunk_plan(desc, cache, true)));
    cudaStream_t st = static_cast<cudaStream_t>(desc->stream);
    const bool bf = desc->dtype == MCSD_DTYPE_BF16;
    if (cache->head_dim == 128) return bf ? launch_chunk<MCSD_DTYPE_BF16, 128>(p, plan, st) : launch_chunk<MCSD_DTYPE_F16, 128>(p, plan, st);
    return bf ? launch_chunk<MCSD_DTYPE_BF16, 64>(p, plan, st) : launch_chunk<MCSD_DTYPE_F16, 64>(p, plan, st);
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
    wait_limits(p);
    const bool mix = mixed(desc);
    cudaStream_t st = static_cast<cudaStream_t>(desc->stream);
    const bool bf = desc->dtype == MCSD_DTYPE_BF16;
    if (cache->head_dim == 128) return bf ? launch_weigh<MCSD_DTYPE_BF16, 128>(p, mix, st) : launch_weigh<MCSD_DTYPE_F16, 128>(p, mix, st);
    return bf ? launch_weigh<MCSD_DTYPE_BF16, 64>(p, mix, st) : launch_weigh<MCSD_DTYPE_F16, 64>(p, mix, st);
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
    if (!on_multiples(4, d->page_table, d->len, d->keep_len, d->weights, d->len_out)) return MCSD_ERR_STRIDE;
    // (what some CTAs read, others must not write)
    const uintptr_t out = reinterpret_cast<uintptr_t>(d->len_out), bytes = 4 * static_cast<uintptr_t>(d->batch);
    for (const int32_t *read : {d->len, d->keep_len}) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(read);
        if (out && at && out < at + bytes && at < out + bytes) return MCSD_ERR_SHAPE;
    }
    if (d->n_layers > (1LL << 40) / (static_cast<int64_t>(d->batch) * cache->n_heads)) return MCSD_ERR_UNSUPPORTED;
    EvictParams p = {};
    p.c = cache_params(cache);
    p.n_layers = d->n_layers; p.layer_stride = d->layer_stride; p.weight_stride = d->weight_stride; p.ld_table = d->ld_table;
    p.table = d->page_table; p.len = d->len; p.keep_len = d->keep_len; p.weights = d->weights; p.len_out = d->len_out;
    p.batch = d->batch; p.max_pages = d->max_pages; p.keep = d->keep; p.sink = d->sink; p.recent = d->recent;
    const long long items = d->n_layers * d->batch * cache->n_heads, room = static_cast<long long>(d->max_pages) * cache->page_size;
    p.n_keys = static_cast<int>(room < kEvictKeys ? room : kEvictKeys);
    const unsigned grid = static_cast<unsigned>(items < 1 << 20 ? items : 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(d->stream);
    if (cache->head_dim == 128) evict_kernel<128><<<grid, kEvictThreads, 4 * p.n_keys, st>>>(p);
    else evict_kernel<64><<<grid, kEvictThreads, 4 * p.n_keys, st>>>(p);
    return launched(1);
}

int mcsd_token_logprobs(const mcsd_logprob_desc *d)
{
    if (!d) return MCSD_ERR_NULL;
    if (d->reserved != 0 || d->vocab < 1 || d->n_given < 0 || d->n_top < 0 || d->n_logits < 0 || d->n_out < 0) return MCSD_ERR_SHAPE;
    if (d->n_top > d->vocab) return MCSD_ERR_SHAPE;
    if (d->vocab > MCSD_MAX_VOCAB || d->n_top > MCSD_MAX_TOP || d->n_out > 0x7fffffffLL) return MCSD_ERR_UNSUPPORTED;
    if (!good_dtype(d->dtype)) return MCSD_ERR_DTYPE;
    if (!(d->temperature > 0.f) || !std::isfinite(d->temperature) || !std::isfinite(1.4426950408889634f / d->temperature)) return MCSD_ERR_TEMPERATURE;
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
    p.scale = 1.4426950408889634f / d->temperature;
    const bool vec = (reinterpret_cast<uintptr_t>(d->logits) | static_cast<unsigned long long>(elem_size(d->dtype)) * static_cast<unsigned long long>(d->ld)) % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(d->stream);
    switch (d->dtype) {
    case MCSD_DTYPE_F32: return launch_logprobs<MCSD_DTYPE_F32>(p, vec, st);
    case MCSD_DTYPE_BF16: return launch_logprobs<MCSD_DTYPE_BF16>(p, vec, st);
    default: return launch_logprobs<MCSD_DTYPE_F16>(p, vec, st);
    }
}

}  // extern "C"
