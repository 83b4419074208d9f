// rules_kernel: penalties for repeated tokens, biases and grammar masks on the logits of a draft tree.
#pragma once

#include "mcsd_common.cuh"

namespace mcsd {

constexpr int kRulesThreads = 256;
constexpr int kRulesMaxSlice = 4096;                // tokens of one CTA
constexpr uint32_t kRulesPrompt = 0x80000000u;      // flag of a counter: the token occurs in the prompt

struct RulesParams {
    const void *logits;
    void *out;
    long long ld_in, ld_out;                        // elements
    const int32_t *history, *history_len, *prompt_len;
    long long ld_history;
    const float *repetition, *frequency, *presence;
    const int32_t *bias_ids;
    const float *bias_values;
    const uint32_t *masks;
    const int32_t *mask_index;
    long long n_masks, ld_mask;
    const int32_t *cand;
    int32_t *status;
    int32_t n_history, n_bias, n_nodes, rows_per_tree, V, slice, node_begin, node_end, rows_per_cta, in_place;
    int16_t parent[MCSD_MAX_NODES];
};

// Adds `step` to the counters of the tokens on the way from node a up to (not including) node `stop`,
// as far as they lie in this CTA's slice.
__device__ __forceinline__ void rules_walk(const RulesParams &P, const int32_t *cand, uint32_t *count, uint32_t *touched,
                                           int x0, int n_el, int a, int stop, uint32_t step)
{
    while (a > stop && a > 0) {
        const uint32_t t = static_cast<uint32_t>(cand[a]) - static_cast<uint32_t>(x0);
        if (t < static_cast<uint32_t>(n_el)) {
            count[t] += step;
            touched[t >> 5] |= 1u << (t & 31);
        }
        a = P.parent[a];
    }
}

// One CTA per (slice of the vocabulary, sequence, run of rows).  It counts the history's tokens that fall
// into its slice in shared memory, once, and then passes over its rows: a token's penalty needs nothing
// but its own counter, so slices never talk to each other, and every CTA scanning the whole history (4
// bytes a token from L2) costs less than a launch that would share the counts.  The tokens on the path
// of a node are added to the same counters before its row and taken out after it: neighbouring rows
// share most of their path, so only the difference of the two paths moves.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kRulesThreads)
rules_kernel(const __grid_constant__ RulesParams P)
{
    using T = Elem<DT>;
    constexpr int VE = 16 / T::kBytes;              // elements of a 16-byte vector
    constexpr int NV = kRulesMaxSlice / (VE * kRulesThreads);
    extern __shared__ uint32_t s_rules[];
    uint32_t *s_count = s_rules;                                            // [slice] occurrences | kRulesPrompt
    float *s_bias = reinterpret_cast<float *>(s_count + P.slice);           // [slice]
    uint32_t *s_touched = reinterpret_cast<uint32_t *>(s_bias + P.slice);   // [slice / 32] tokens a rule concerns
    int32_t *s_cand = reinterpret_cast<int32_t *>(s_touched + P.slice / 32);// [n_nodes]
    const int tid = threadIdx.x, b = blockIdx.y;
    const int x0 = blockIdx.x * P.slice;
    const int n_el = min(P.slice, P.V - x0);
    const bool penalise = P.repetition || P.frequency || P.presence;

    int32_t *s_index = reinterpret_cast<int32_t *>(s_bias);
    for (int i = tid; i < P.slice; i += kRulesThreads) { s_count[i] = 0u; s_index[i] = 0; }
    if (penalise && P.cand)
        for (int i = tid; i < P.n_nodes; i += kRulesThreads) s_cand[i] = P.cand[static_cast<long long>(b) * P.n_nodes + i];
    __syncthreads();
    if (penalise && P.history) {
        const int32_t *row = P.history + b * P.ld_history;
        const int len = min(max(P.history_len[b], 0), P.n_history);
        const int prompt = P.prompt_len ? P.prompt_len[b] : 0;
        for (int i = tid; i < len; i += kRulesThreads) {
            const uint32_t t = static_cast<uint32_t>(row[i]) - static_cast<uint32_t>(x0);
            if (t < static_cast<uint32_t>(n_el)) {    // (false for negative tokens as well)
                if (i < prompt) atomicOr(&s_count[t], kRulesPrompt);
                else atomicAdd(&s_count[t], 1u);
            }
        }
    }
    for (int i = tid; i < P.n_bias; i += kRulesThreads) {
        const uint32_t t = static_cast<uint32_t>(P.bias_ids[static_cast<long long>(b) * P.n_bias + i]) - static_cast<uint32_t>(x0);
        if (t < static_cast<uint32_t>(n_el)) atomicMax(&s_index[t], i + 1);   // the highest entry counts
    }
    __syncthreads();
    for (int i = tid; i < P.slice; i += kRulesThreads) {                     // (slice: a multiple of the CTA's threads)
        const int at = s_index[i];
        const float v = at ? P.bias_values[static_cast<long long>(b) * P.n_bias + at - 1] : 0.f;
        s_bias[i] = v;
        const uint32_t any = __ballot_sync(0xffffffffu, v != 0.f || s_count[i] != 0u);
        if ((tid & 31) == 0) s_touched[i >> 5] = any;
    }
    const float theta = P.repetition ? P.repetition[b] : 1.f;
    const float freq = P.frequency ? P.frequency[b] : 0.f;
    const float pres = P.presence ? P.presence[b] : 0.f;

    auto apply = [&](float l, int i) {
        const uint32_t c = s_count[i], n = c & ~kRulesPrompt;
        if (c) l = l > 0.f ? l / theta : l * theta;
        if (n) l = l - freq * static_cast<float>(n) - pres;
        const float v = s_bias[i];
        return v != 0.f ? l + v : l;
    };

    int before = 0;                                  // node whose path is in the counters
    const int n0 = P.node_begin + blockIdx.z * P.rows_per_cta;
    const int n1 = min(n0 + P.rows_per_cta, P.node_end);
    for (int n = n0; n < n1; ++n) {
        __syncthreads();                             // the row before is done with the counters
        if (tid == 0 && penalise && P.cand) {
            int a = before, c = n;                   // their lowest common ancestor
            while (a != c) {
                if (a > c) a = P.parent[a]; else c = P.parent[c];
            }
            rules_walk(P, s_cand, s_count, s_touched, x0, n_el, before, a, 0xffffffffu);
            rules_walk(P, s_cand, s_count, s_touched, x0, n_el, n, a, 1u);
        }
        before = n;
        const long long r = static_cast<long long>(b) * P.rows_per_tree + n;
        const uint32_t *mask = nullptr;
        if (P.masks) {
            const long long item = static_cast<long long>(b) * P.n_nodes + n;
            const long long m = P.mask_index ? P.mask_index[item] : item;
            if (m >= 0 && m < P.n_masks) mask = P.masks + m * P.ld_mask + (x0 >> 5);
            else if (m >= 0 && P.status && blockIdx.x == 0 && tid == 0) atomicOr(&P.status[b], MCSD_STATUS_BAD_MASK);
        }
        __syncthreads();
        const char *src = static_cast<const char *>(P.logits) + (r * P.ld_in + x0) * T::kBytes;
        char *dst = static_cast<char *>(P.out) + (r * P.ld_out + x0) * T::kBytes;
        if constexpr (VEC) {
            uint4 v[NV];
            uint32_t keep[NV], hit[NV];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int i = (tid + k * kRulesThreads) * VE;
                keep[k] = (1u << VE) - 1u;
                hit[k] = 0u;
                if (i + VE <= n_el) {
                    if (mask) keep[k] &= __ldg(mask + (i >> 5)) >> (i & 31);
                    hit[k] = (s_touched[i >> 5] >> (i & 31)) & ((1u << VE) - 1u);
                }
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int i = (tid + k * kRulesThreads) * VE;
                // in place a vector that no rule concerns is not read, nor one that is masked as a whole
                const bool rd = i + VE <= n_el && keep[k] != 0u && (!P.in_place || hit[k] || keep[k] != (1u << VE) - 1u);
                v[k] = ld_plain_v4_if(src + static_cast<long long>(i) * T::kBytes, rd);
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int i = (tid + k * kRulesThreads) * VE;
                if (i + VE > n_el) continue;
                if (P.in_place && !hit[k] && keep[k] == (1u << VE) - 1u) continue;
                if (hit[k] || keep[k] != (1u << VE) - 1u) {
                    float f[VE];
                    T::unpack(v[k], f);
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        if ((hit[k] >> e) & 1u) f[e] = apply(f[e], i + e);
                        if (!((keep[k] >> e) & 1u)) f[e] = -INFINITY;
                    }
                    v[k] = pack_elems<DT>(f);
                }
                *reinterpret_cast<uint4 *>(dst + static_cast<long long>(i) * T::kBytes) = v[k];
            }
            const int tail = n_el & ~(VE - 1);       // the last tokens of the vocabulary, one by one
            if (tid < n_el - tail) {
                const int i = tail + tid;
                float l = apply(load_elem<DT>(src, i), i);
                if (mask && !((mask[i >> 5] >> (i & 31)) & 1u)) l = -INFINITY;
                store_elem<DT>(dst, i, l);
            }
        } else {
            for (int i = tid; i < n_el; i += kRulesThreads) {
                float l = apply(load_elem<DT>(src, i), i);
                if (mask && !((mask[i >> 5] >> (i & 31)) & 1u)) l = -INFINITY;
                store_elem<DT>(dst, i, l);
            }
        }
    }
}

}  // namespace mcsd
