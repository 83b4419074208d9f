// Host side of the operators around the verification step: argument validation, launch configuration
// and the extern "C" entry points from mcsd_apply_logit_rules on (mcsd.h).
#include <cmath>

#include "mcsd_common.cuh"
#include "mcsd_rules.cuh"
#include "mcsd_pages.cuh"
#include "mcsd_cache.cuh"
#include "mcsd_attend.cuh"
#include "mcsd_attend_wide.cuh"
#include "mcsd_launch.cuh"

namespace mcsd {
namespace {

// ---- logit rules
template <int DT>
int launch_rules(const RulesParams &p, dim3 grid, size_t smem, bool vec, cudaStream_t st)
{
    // (trees some hundred levels deep; the kernel's own static part counts against the default of 48 KB as well)
    const int more = smem > 40000 ? static_cast<int>(smem) : 0;
    if (vec) {
        if (more && !allow_smem<rules_kernel<DT, true>>(more)) return MCSD_ERR_CUDA;
        rules_kernel<DT, true><<<grid, kRulesThreads, smem, st>>>(p);
    } else {
        if (more && !allow_smem<rules_kernel<DT, false>>(more)) return MCSD_ERR_CUDA;
        rules_kernel<DT, false><<<grid, kRulesThreads, smem, st>>>(p);
    }
    return launched(1);
}

// ---- rows of the cache
template <bool APPEND, int DT, int D>
int launch_rows(const RowsParams &p, bool vec, cudaStream_t st)
{
    // A group of D / 8 threads per row (2 n_heads groups a token) while that fills the SMs, then several tokens a
    // group; a token at least.
    const long long groups = 256 / (D / 8), rows = 2LL * p.c.n_heads, resident = static_cast<long long>(sm_count()) * (APPEND ? kAppendCtas : kReadCtas);
    if (resident <= 0) return MCSD_ERR_CUDA;
    const long long want = (p.n_tokens * rows + groups - 1) / groups, least = (rows + groups - 1) / groups;
    const long long cap = resident > least ? resident : least;
    const unsigned grid = static_cast<unsigned>(want < cap ? want : cap);
    if constexpr (APPEND) {
        if (vec) append_kernel<DT, D, true><<<grid, 256, 0, st>>>(p);
        else append_kernel<DT, D, false><<<grid, 256, 0, st>>>(p);
    } else {
        if (vec) read_kernel<DT, D, true><<<grid, 256, 0, st>>>(p);
        else read_kernel<DT, D, false><<<grid, 256, 0, st>>>(p);
    }
    return launched(1);
}

template <bool APPEND>
int rows_call(const mcsd_kv_cache *cache, const void *keys, int64_t key_token, int64_t key_head, const void *values,
              int64_t value_token, int64_t value_head, int32_t dtype, int64_t n_tokens, const int64_t *slots, void *stream)
{
    const int rc = check_cache(cache);
    if (rc != MCSD_OK) return rc;
    if (!good_dtype(dtype)) return MCSD_ERR_DTYPE;
    if (n_tokens < 0) return MCSD_ERR_SHAPE;
    if (key_token < 0 || value_token < 0 || key_head < 0 || value_head < 0) return MCSD_ERR_STRIDE;
    set_last_launches(0);
    if (n_tokens == 0 || cache->n_pages == 0) return MCSD_OK;
    if (!slots || (APPEND ? !keys || !values : !keys && !values)) return MCSD_ERR_NULL;
    if (!on_multiples(static_cast<unsigned>(elem_size(dtype)), keys, values) || !on_multiples(8, slots)) return MCSD_ERR_STRIDE;
    const int64_t row = cache->head_dim;
    // rows must not overlap where they are written
    if (!APPEND && ((keys && cache->n_heads > 1 && key_head < row) || (values && cache->n_heads > 1 && value_head < row))) return MCSD_ERR_STRIDE;
    if (!APPEND && n_tokens > 1 && ((keys && key_token < row) || (values && value_token < row))) return MCSD_ERR_STRIDE;
    if (n_tokens > (1LL << 40) / cache->n_heads) return MCSD_ERR_UNSUPPORTED;
    RowsParams p = {};
    p.c = cache_params(cache);
    p.keys = const_cast<void *>(keys);
    p.values = const_cast<void *>(values);
    p.key_token = key_token; p.key_head = key_head; p.value_token = value_token; p.value_head = value_head;
    p.slots = reinterpret_cast<const long long *>(slots);
    p.n_tokens = n_tokens;
    const unsigned long long es = static_cast<unsigned long long>(elem_size(dtype));
    const unsigned long long all = reinterpret_cast<uintptr_t>(keys) | reinterpret_cast<uintptr_t>(values) |
        es * static_cast<unsigned long long>(key_token | key_head | value_token | value_head);
    const bool vec = all % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cache->head_dim == 128) {
        switch (dtype) {
        case MCSD_DTYPE_F32: return launch_rows<APPEND, MCSD_DTYPE_F32, 128>(p, vec, st);
        case MCSD_DTYPE_BF16: return launch_rows<APPEND, MCSD_DTYPE_BF16, 128>(p, vec, st);
        default: return launch_rows<APPEND, MCSD_DTYPE_F16, 128>(p, vec, st);
        }
    }
    switch (dtype) {
    case MCSD_DTYPE_F32: return launch_rows<APPEND, MCSD_DTYPE_F32, 64>(p, vec, st);
    case MCSD_DTYPE_BF16: return launch_rows<APPEND, MCSD_DTYPE_BF16, 64>(p, vec, st);
    default: return launch_rows<APPEND, MCSD_DTYPE_F16, 64>(p, vec, st);
    }
}

// ---- tree attention
int check_attention(const mcsd_attention_desc *d, const mcsd_kv_cache *cache)
{
    if (!d) return MCSD_ERR_NULL;
    const int rc = check_cache(cache);
    if (rc != MCSD_OK) return rc;
    if (d->reserved != 0 || d->batch < 0 || d->n_nodes < 1 || d->n_heads < 1 || d->max_pages < 0) return MCSD_ERR_SHAPE;
    if (d->n_heads % cache->n_heads != 0) return MCSD_ERR_SHAPE;
    if (d->n_nodes > MCSD_MAX_NODES) return MCSD_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d->max_pages) * cache->page_size > 0x7fffffffLL - MCSD_MAX_NODES) return MCSD_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d->batch) * d->n_nodes * d->n_heads > 0x7fffffffLL) return MCSD_ERR_UNSUPPORTED;
    if (d->dtype != MCSD_DTYPE_BF16 && d->dtype != MCSD_DTYPE_F16) return MCSD_ERR_DTYPE;
    if (d->ld_table < d->max_pages) return MCSD_ERR_STRIDE;
    if (d->q_seq_stride < 0 || d->q_node_stride < 0 || d->q_head_stride < 0) return MCSD_ERR_STRIDE;
    const int64_t row = cache->head_dim;
    if ((d->n_heads > 1 && d->out_head_stride < row) || (d->n_nodes > 1 && d->out_node_stride < row) ||
        (d->batch > 1 && d->out_seq_stride < row) || d->out_head_stride < 0 || d->out_node_stride < 0 || d->out_seq_stride < 0)
        return MCSD_ERR_STRIDE;
    return MCSD_OK;
}

// How a call is laid out; depends on the sizes only.
struct AttentionPlan {
    int rows;       // rows of a block
    int blocks;     // blocks per key/value head
    int lead;       // places of the cut an item costs beside its units
    int ctas;       // CTAs the work is cut for: what is resident at once, or one per unit where a call cannot have more
};
AttentionPlan attention_plan(const mcsd_attention_desc *d, const mcsd_kv_cache *cache)
{
    AttentionPlan plan;
    int sms = sm_count();
    if (sms <= 0) sms = 148;
    const long long rows = static_cast<long long>(d->n_nodes) * (d->n_heads / cache->n_heads);
    // Blocks of 8, 16 and 24 rows decode the keys again for every block (24 rows leave two CTAs per SM instead of three
    // or four), one of 128 takes about as long for few rows as for all.  Measured (128 numbers a head, 8 sequences x 32
    // key heads x 2000 positions | 4 sequences x 8 key heads x 16000 positions, us):
    //   rows   blocks of 16   blocks of 24   one of 128
    //   24     69 | 66        52 | 52        86 | 77
    //   32     70 | 66        85 | 76        87 | 76
    //   45     99 | 89        88 | 78        87 | 76
    //   60     124 | 109      121 | 105      97 | 78
    plan.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 24 ? 24 : rows <= 32 ? 16 : rows <= 48 ? 24 : kWideRows;
    plan.blocks = static_cast<int>((rows + plan.rows - 1) / plan.rows);
    // Measured for 0, 1, 2, 3, 4, 6, 8 and 12 places an item: decoding is fastest with 2 or 3, blocks of 16 and 24 rows with 3 to 8,
    // those of 128 rows with 4 to 6 for a tree of 45 nodes and 6 to 8 for one of 181 (its units see masks); 2 places off costs 2 %.
    plan.lead = plan.rows == 8 ? 2 : plan.rows < kWideRows ? 4 : 4 + 2 * ((d->n_nodes + kAttUnit - 1) / kAttUnit);
    const long long units = (static_cast<long long>(d->max_pages) * cache->page_size + kAttUnit - 1) / kAttUnit;
    const long long most = static_cast<long long>(d->batch) * cache->n_heads * plan.blocks * (units > 0 ? units : 1);
    const long long resident = static_cast<long long>(plan.rows == 8 ? kNarrowCtas<1> : plan.rows == 16 ? kNarrowCtas<2> : plan.rows == 24 ? kNarrowCtas<3> : 1) * sms;
    plan.ctas = static_cast<int>(most < 1 ? 1 : most < resident ? most : resident);
    return plan;
}

// Launches the kernel that does the work and, as its programmatic dependent, the one that joins divided items.
template <int DT, int D, int ROWS, auto Kernel>
int launch_with_join(int threads, int smem, const AttendParams &p, cudaStream_t st)
{
    if (!allow_smem<Kernel>(smem)) return MCSD_ERR_CUDA;
    Kernel<<<p.n_ctas, threads, smem, st>>>(p);
    if (cudaGetLastError() != cudaSuccess) return MCSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.batch * p.c.n_heads * p.n_blocks), ROWS / 8);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, join_kernel<DT, D, ROWS>, p) != cudaSuccess) return MCSD_ERR_CUDA;
    return launched(2);
}

template <int DT, int D>
int launch_attention(const AttendParams &p, int rows, cudaStream_t st)
{
    if (rows == 8) return launch_with_join<DT, D, 8, narrow_kernel<DT, D, 1, TreeRows>>(kNarrowWarps * 32, kNarrowSmem<D, 1>, p, st);
    if (rows == 16) return launch_with_join<DT, D, 16, narrow_kernel<DT, D, 2, TreeRows>>(kNarrowWarps * 32, kNarrowSmem<D, 2>, p, st);
    if (rows == 24) return launch_with_join<DT, D, 24, narrow_kernel<DT, D, 3, TreeRows>>(kNarrowWarps * 32, kNarrowSmem<D, 3>, p, st);
    return launch_with_join<DT, D, kWideRows, wide_kernel<DT, D>>(kWideThreads, kWideSmem<D>, p, st);
}

}  // namespace
}  // namespace mcsd

using namespace mcsd;

extern "C" {

int mcsd_apply_logit_rules(const mcsd_desc *desc, const mcsd_logit_rules *rules, const int32_t *tree_parent,
                           const int32_t *cand_tokens, const void *logits, int64_t ld_in, void *out, int64_t ld_out,
                           int32_t rows_per_tree, int32_t node_begin, int32_t node_end)
{
    if (!desc || !rules) return MCSD_ERR_NULL;
    if (desc->reserved != 0 || desc->batch < 0 || desc->n_nodes < 1 || desc->vocab < 1) return MCSD_ERR_SHAPE;
    if (desc->n_nodes > MCSD_MAX_NODES || desc->vocab > MCSD_MAX_VOCAB || desc->batch > 65535) return MCSD_ERR_UNSUPPORTED;
    if (!good_dtype(desc->dtype)) return MCSD_ERR_DTYPE;
    if (!tree_parent) return MCSD_ERR_NULL;
    const int depth = tree_depth(tree_parent, desc->n_nodes);
    if (depth < 0) return depth;
    if (rows_per_tree < 0 || rows_per_tree > desc->n_nodes || node_begin < 0 || node_end > rows_per_tree || node_begin > node_end)
        return MCSD_ERR_SHAPE;
    if (ld_in < desc->vocab || ld_out < desc->vocab) return MCSD_ERR_STRIDE;
    if (rules->n_bias < 0 || rules->n_history < 0 || rules->n_masks < 0) return MCSD_ERR_SHAPE;
    if (rules->history && rules->ld_history < rules->n_history) return MCSD_ERR_STRIDE;
    if (rules->masks && rules->ld_mask < (desc->vocab + 31) / 32) return MCSD_ERR_STRIDE;
    if (rules->history && !rules->history_len) return MCSD_ERR_NULL;
    if (rules->n_bias > 0 && (!rules->bias_ids != !rules->bias_values)) return MCSD_ERR_NULL;
    set_last_launches(0);
    const int n_rows = node_end - node_begin;
    if (desc->batch == 0 || n_rows == 0) return MCSD_OK;
    if (!logits || !out) return MCSD_ERR_NULL;
    if (logits == out && ld_in != ld_out) return MCSD_ERR_STRIDE;
    if (!on_multiples(static_cast<unsigned>(elem_size(desc->dtype)), logits, out) ||
        !on_multiples(4, cand_tokens, desc->out_status, rules->history, rules->history_len, rules->prompt_len, rules->repetition, rules->frequency,
                      rules->presence, rules->bias_ids, rules->bias_values, rules->masks, rules->mask_index))
        return MCSD_ERR_STRIDE;
    const bool penalise = rules->repetition || rules->frequency || rules->presence;
    if (penalise && !cand_tokens && depth > 0) return MCSD_ERR_NULL;

    RulesParams p = {};
    p.logits = logits; p.out = out; p.ld_in = ld_in; p.ld_out = ld_out;
    p.history = rules->history; p.history_len = rules->history_len; p.prompt_len = rules->prompt_len;
    p.ld_history = rules->ld_history; p.n_history = rules->n_history;
    p.repetition = rules->repetition; p.frequency = rules->frequency; p.presence = rules->presence;
    p.bias_ids = rules->bias_ids; p.bias_values = rules->bias_values;
    p.n_bias = rules->bias_ids ? rules->n_bias : 0;
    p.masks = rules->masks; p.mask_index = rules->mask_index; p.n_masks = rules->n_masks; p.ld_mask = rules->ld_mask;
    p.cand = cand_tokens; p.status = desc->out_status;
    p.n_nodes = desc->n_nodes; p.rows_per_tree = rows_per_tree; p.V = desc->vocab;
    p.node_begin = node_begin; p.node_end = node_end; p.in_place = logits == out;
    for (int n = 0; n < desc->n_nodes; ++n) p.parent[n] = static_cast<int16_t>(tree_parent[n]);
    const int sms = sm_count();
    if (sms <= 0) return MCSD_ERR_CUDA;
    // The widest slice (fewest scans of the history) that still gives every SM two CTAs, rows split
    // where a narrow slice alone does not; a CTA has eight warps, a row each.
    p.depth = depth;
    p.slice = kRulesMaxSlice;
    while (p.slice > 512 && static_cast<long long>((p.V + p.slice - 1) / p.slice) * desc->batch < 2LL * sms) p.slice >>= 1;
    const long long ctas = static_cast<long long>((p.V + p.slice - 1) / p.slice) * desc->batch;
    long long split = (4LL * sms + ctas - 1) / ctas;
    if (split > (n_rows + 7) / 8) split = (n_rows + 7) / 8;
    p.rows_per_cta = static_cast<int32_t>((n_rows + split - 1) / split);
    const dim3 grid((p.V + p.slice - 1) / p.slice, desc->batch, (n_rows + p.rows_per_cta - 1) / p.rows_per_cta);
    const size_t smem = 4 * (2 * static_cast<size_t>(p.slice) + p.slice / 2 + p.slice / 32 + desc->n_nodes + kRulesThreads / 32 * 2 * static_cast<size_t>(depth));
    const unsigned long long es = static_cast<unsigned long long>(elem_size(desc->dtype));
    const bool vec = (reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out) |
                      es * static_cast<unsigned long long>(ld_in | ld_out)) % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(desc->stream);
    switch (desc->dtype) {
    case MCSD_DTYPE_F32: return launch_rules<MCSD_DTYPE_F32>(p, grid, smem, vec, st);
    case MCSD_DTYPE_BF16: return launch_rules<MCSD_DTYPE_BF16>(p, grid, smem, vec, st);
    default: return launch_rules<MCSD_DTYPE_F16>(p, grid, smem, vec, st);
    }
}

int mcsd_build_page_tables(const mcsd_page_desc *d)
{
    if (!d) return MCSD_ERR_NULL;
    if (d->reserved != 0 || d->batch < 0 || d->max_pages < 0 || d->new_tokens < 0 || d->ring_capacity < 0 || d->n_slots < 0)
        return MCSD_ERR_SHAPE;
    if (d->batch > 0 && d->ring_capacity == 0) return MCSD_ERR_SHAPE;
    if (!good_page_size(d->page_size) || d->batch > MCSD_MAX_SEQUENCES) return MCSD_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d->max_pages) * d->page_size > 0x7fffffffLL) return MCSD_ERR_UNSUPPORTED;
    if (d->ld_table < d->max_pages) return MCSD_ERR_STRIDE;
    set_last_launches(0);
    if (d->batch == 0) return MCSD_OK;
    if (!d->start || !d->held || !d->ring_state || !d->ring || (!d->page_table && d->max_pages > 0))
        return MCSD_ERR_NULL;
    if (!on_multiples(4, d->start, d->count, d->page_table, d->held, d->held_out, d->ring, d->ring_state, d->ring_state_out, d->cu_tokens, d->status) ||
        !on_multiples(8, d->slots))
        return MCSD_ERR_STRIDE;
    PagesParams p = {};
    p.start = d->start; p.count = d->count; p.table = d->page_table;
    p.held = d->held; p.held_out = d->held_out ? d->held_out : d->held;
    p.ring = d->ring; p.state = d->ring_state; p.state_out = d->ring_state_out ? d->ring_state_out : d->ring_state;
    p.slots = reinterpret_cast<long long *>(d->slots);
    p.cu_tokens = d->cu_tokens; p.status = d->status;
    p.ld_table = d->ld_table; p.n_slots = d->slots ? d->n_slots : 0;
    p.batch = d->batch; p.page_shift = shift_of(d->page_size); p.max_pages = d->max_pages; p.new_tokens = d->new_tokens;
    p.cap = d->ring_capacity;
    p.commit_last = p.held_out == p.held || p.state_out == p.state;
    const int sms = sm_count();
    if (sms <= 0) return MCSD_ERR_CUDA;
    // one CTA per 2048 slots or 32 sequences, one per SM at most
    long long ctas = (p.n_slots + 2047) / 2048;
    if (ctas < (d->batch + 31) / 32) ctas = (d->batch + 31) / 32;
    if (ctas > sms) ctas = sms;
    const size_t smem = sizeof(int32_t) * (5 * static_cast<size_t>(d->batch) + 1);
    if (smem > 40000 && !allow_smem<pages_kernel>(static_cast<int>(smem))) return MCSD_ERR_CUDA;
    pages_kernel<<<static_cast<unsigned>(ctas), kPagesThreads, smem, static_cast<cudaStream_t>(d->stream)>>>(p);
    return launched(1);
}

size_t mcsd_kv_block_bytes(int32_t head_dim, int32_t page_size)
{
    if ((head_dim != 64 && head_dim != 128) || !good_page_size(page_size)) return 0;
    return static_cast<size_t>(kv_block_bytes(head_dim, page_size));
}

int mcsd_append_kv(const mcsd_kv_cache *cache, const void *keys, int64_t key_token_stride, int64_t key_head_stride,
                   const void *values, int64_t value_token_stride, int64_t value_head_stride, int32_t dtype,
                   int64_t n_tokens, const int64_t *slots, void *stream)
{
    return rows_call<true>(cache, keys, key_token_stride, key_head_stride, values, value_token_stride, value_head_stride, dtype,
                           n_tokens, slots, stream);
}

int mcsd_read_kv(const mcsd_kv_cache *cache, void *keys, int64_t key_token_stride, int64_t key_head_stride, void *values,
                 int64_t value_token_stride, int64_t value_head_stride, int32_t dtype, int64_t n_tokens, const int64_t *slots,
                 void *stream)
{
    return rows_call<false>(cache, keys, key_token_stride, key_head_stride, values, value_token_stride, value_head_stride, dtype,
                            n_tokens, slots, stream);
}

size_t mcsd_tree_attention_workspace_bytes(const mcsd_attention_desc *desc, const mcsd_kv_cache *cache)
{
    if (check_attention(desc, cache) != MCSD_OK) return 0;
    const AttentionPlan plan = attention_plan(desc, cache);
    return (2 * sizeof(float) * part_floats(plan.rows, cache->head_dim) * static_cast<size_t>(plan.ctas) + 255) / 256 * 256;
}

int mcsd_tree_attention(const mcsd_attention_desc *desc, const mcsd_kv_cache *cache, const int32_t *page_table,
                        const int32_t *prefix_len, const int32_t *tree_parent, const void *q, void *out, float *lse)
{
    const int rc = check_attention(desc, cache);
    if (rc != MCSD_OK) return rc;
    if (!tree_parent) return MCSD_ERR_NULL;
    const int depth = tree_depth(tree_parent, desc->n_nodes);
    if (depth < 0) return depth;
    if (!std::isfinite(desc->scale)) return MCSD_ERR_SHAPE;
    set_last_launches(0);
    if (desc->batch == 0) return MCSD_OK;
    if (!prefix_len || !q || !out || (!page_table && desc->max_pages > 0)) return MCSD_ERR_NULL;
    if (!on_multiples(2, q, out) || !on_multiples(4, page_table, prefix_len, lse)) return MCSD_ERR_STRIDE;
    if (!desc->workspace || reinterpret_cast<uintptr_t>(desc->workspace) % 256 != 0 ||
        desc->workspace_bytes < mcsd_tree_attention_workspace_bytes(desc, cache))
        return MCSD_ERR_WORKSPACE;
    const AttentionPlan plan = attention_plan(desc, cache);
    // (the cut counts units of all items, and what stands for the items themselves, in 32 bits)
    if (static_cast<double>(desc->batch) * cache->n_heads * plan.blocks *
            (static_cast<double>(desc->max_pages) * cache->page_size / kAttUnit + 2 + plan.lead) > 4.2e9)
        return MCSD_ERR_UNSUPPORTED;
    AttendParams p = {};
    p.c = cache_params(cache);
    p.q = q; p.out = out; p.lse = lse; p.table = page_table; p.prefix_len = prefix_len; p.ld_table = desc->ld_table;
    p.q_seq = desc->q_seq_stride; p.q_node = desc->q_node_stride; p.q_head = desc->q_head_stride;
    p.o_seq = desc->out_seq_stride; p.o_node = desc->out_node_stride; p.o_head = desc->out_head_stride;
    p.batch = desc->batch; p.n_nodes = desc->n_nodes; p.n_heads = desc->n_heads; p.max_pages = desc->max_pages;
    p.scale = desc->scale;
    p.scale_part = scale_part(desc->scale, &p.scale_power);
    const int polls = mcsd_get_option(MCSD_OPT_WAIT_POLLS);
    p.wait_polls = polls > 0 ? static_cast<uint32_t>(polls) : kWaitPolls;
    p.test_extra = mcsd_get_option(MCSD_OPT_TEST_EXTRA_TX) > 0 ? 1u : 0u;
    for (int n = 0; n < desc->n_nodes; ++n) p.parent[n] = static_cast<int16_t>(tree_parent[n]);
    p.group = desc->n_heads / cache->n_heads;
    p.n_rows = desc->n_nodes * p.group;
    p.n_blocks = plan.blocks;
    p.n_ctas = plan.ctas;
    p.lead = static_cast<uint32_t>(plan.lead);
    p.part = static_cast<float *>(desc->workspace);
    p.q_vec = (reinterpret_cast<uintptr_t>(q) | 2ull * static_cast<unsigned long long>(desc->q_seq_stride | desc->q_node_stride |
                                                                                       desc->q_head_stride)) % 16 == 0;
    p.o_vec = (reinterpret_cast<uintptr_t>(out) | 2ull * static_cast<unsigned long long>(desc->out_seq_stride | desc->out_node_stride |
                                                                                         desc->out_head_stride)) % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(desc->stream);
    const bool bf = desc->dtype == MCSD_DTYPE_BF16;
    if (cache->head_dim == 128) return bf ? launch_attention<MCSD_DTYPE_BF16, 128>(p, plan.rows, st) : launch_attention<MCSD_DTYPE_F16, 128>(p, plan.rows, st);
    return bf ? launch_attention<MCSD_DTYPE_BF16, 64>(p, plan.rows, st) : launch_attention<MCSD_DTYPE_F16, 64>(p, plan.rows, st);
}

int mcsd_gather_accepted_pages(const mcsd_kv_cache *cache, int64_t n_layers, int64_t layer_stride, const int32_t *page_table,
                               int64_t ld_table, int32_t max_pages, int32_t batch, const int32_t *prefix_len,
                               const int32_t *path_nodes, const int32_t *accept_len, int32_t gamma, void *stream)
{
    const int rc = check_cache(cache);
    if (rc != MCSD_OK) return rc;
    if (n_layers < 0 || batch < 0 || gamma < 0 || max_pages < 0) return MCSD_ERR_SHAPE;
    if (ld_table < max_pages || layer_stride % 16 != 0 || layer_stride < 0) return MCSD_ERR_STRIDE;
    if (n_layers > 1 && layer_stride < static_cast<int64_t>(mcsd_kv_block_bytes(cache->head_dim, cache->page_size)) * cache->n_heads)
        return MCSD_ERR_STRIDE;
    set_last_launches(0);
    if (n_layers == 0 || batch == 0 || gamma == 0 || max_pages == 0 || cache->n_pages == 0) return MCSD_OK;
    if (!page_table || !prefix_len || !path_nodes || !accept_len) return MCSD_ERR_NULL;
    if (!on_multiples(4, page_table, prefix_len, path_nodes, accept_len)) return MCSD_ERR_STRIDE;
    if (n_layers > (1LL << 40) / (static_cast<int64_t>(batch) * cache->n_heads)) return MCSD_ERR_UNSUPPORTED;
    MoveParams p = {};
    p.c = cache_params(cache);
    p.n_layers = n_layers; p.layer_stride = layer_stride;
    p.table = page_table; p.prefix_len = prefix_len; p.path_nodes = path_nodes; p.accept_len = accept_len;
    p.ld_table = ld_table; p.max_pages = max_pages; p.batch = batch; p.gamma = gamma;
    // runs of layers as long as the threads of four CTAs per SM still have one each, up to eight
    const long long cap = static_cast<long long>(sm_count()) * 8, lines = static_cast<long long>(batch) * cache->n_heads;
    if (cap <= 0) return MCSD_ERR_CUDA;
    long long run = n_layers * lines / (cap / 2 * 16);
    run = run < 1 ? 1 : run > 8 ? 8 : run;
    p.layers_per_item = static_cast<int32_t>(run);
    const long long want = ((n_layers + run - 1) / run * lines + 15) / 16;
    const unsigned grid = static_cast<unsigned>(want < cap ? want : cap);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cache->head_dim == 128) move_kernel<128><<<grid, 256, 0, st>>>(p);
    else move_kernel<64><<<grid, 256, 0, st>>>(p);
    return launched(1);
}

}  // extern "C"
