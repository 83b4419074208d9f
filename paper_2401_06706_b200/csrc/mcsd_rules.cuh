// rules_kernel: penalties for repeated tokens, biases and grammar masks on the logits of a draft tree.
#pragma once

#include "mcsd_common.cuh"

namespace mcsd {

constexpr int kRulesThreads = 256;
constexpr int kRulesMaxSlice = 2048;                // tokens of one CTA: four CTAs per SM
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
    int32_t depth;                                  // of the tree: the longest path, the root excluded
    int16_t parent[MCSD_MAX_NODES];
};

// One CTA per (slice of the vocabulary, sequence, run of rows).  It counts the history's tokens that fall
// into its slice in shared memory, once: a token's penalty needs nothing but its own counter, so slices
// never talk to each other, and every CTA scanning the whole history (4 bytes a token from L2) costs less
// than a launch that would share the counts.  Then every warp takes rows of its own, without a barrier: it
// streams its slice of the row (eight 16-byte loads in flight per lane) with nothing but the mask applied, then
// takes the tokens some rule concerns one by one from a list, and last the few on the row's path, from their
// logits read before.  (With the rules applied while streaming, nearly every warp had a lane with a token
// that needs them, and all lanes went through them: 215 us against 137 us on 64 x 31 rows of 50272 halves; the mask's words taken by shuffles from one load a
// lane and four CTAs per SM instead of three made that 108 us, 3.7 TB/s or 0.56 of the measured copy bandwidth.
// What is left: a CTA asks for its first row behind five dependent loads and four barriers, and a warp for its next row when it is through
// with one. In place the same takes 115 us, without masks 48 us.)
template <int DT, bool VEC>
__global__ void __launch_bounds__(kRulesThreads, 4)
rules_kernel(const __grid_constant__ RulesParams P)
{
    using T = Elem<DT>;
    constexpr int VE = 16 / T::kBytes;              // elements of a 16-byte vector
    constexpr uint32_t kAll = (1u << VE) - 1u;
    constexpr int kFlight = 8, kWarps = kRulesThreads / 32;
    extern __shared__ uint32_t s_rules[];
    uint32_t *s_count = s_rules;                                            // [slice] occurrences | kRulesPrompt
    float *s_bias = reinterpret_cast<float *>(s_count + P.slice);           // [slice]
    uint32_t *s_touched = reinterpret_cast<uint32_t *>(s_bias + P.slice);   // [slice / 32] tokens a rule concerns
    uint16_t *s_list = reinterpret_cast<uint16_t *>(s_touched + P.slice / 32); // [slice] these tokens in ascending order
    int32_t *s_cand = reinterpret_cast<int32_t *>(s_list + P.slice);        // [n_nodes]
    __shared__ int s_listed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.y;
    int32_t *s_token = s_cand + P.n_nodes + warp * 2 * P.depth;             // [depth] tokens on the path of this warp's row
    float *s_value = reinterpret_cast<float *>(s_token + P.depth);          // [depth] their logits
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
#pragma unroll 4
        for (int i = tid; i < len; i += kRulesThreads) {
            const uint32_t t = static_cast<uint32_t>(__ldg(row + i)) - static_cast<uint32_t>(x0);
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
        if (lane == 0) s_touched[i >> 5] = any;
    }
    const float theta = P.repetition ? P.repetition[b] : 1.f;
    const float freq = P.frequency ? P.frequency[b] : 0.f;
    const float pres = P.presence ? P.presence[b] : 0.f;
    __syncthreads();
    if (warp == 0) {
        const int per = P.slice / 1024;              // words of the bitmap per lane (slice: at least 512, half of the lanes then)
        int n = 0;
        for (int w = lane * max(per, 1); w < (lane + 1) * max(per, 1) && w < P.slice / 32; ++w) n += __popc(s_touched[w]);
        int at = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, at, o);
            if (lane >= o) at += t;
        }
        if (lane == 31) s_listed = at;
        at -= n;
        for (int w = lane * max(per, 1); w < (lane + 1) * max(per, 1) && w < P.slice / 32; ++w)
            for (uint32_t bits = s_touched[w]; bits; bits &= bits - 1u) s_list[at++] = static_cast<uint16_t>(32 * w + __ffs(bits) - 1);
    }
    __syncthreads();
    const int listed = s_listed;

    // the rules but the mask; c: occurrences | kRulesPrompt
    auto apply = [&](float l, uint32_t c, float v) {
        const uint32_t n = c & ~kRulesPrompt;
        if (c) l = l > 0.f ? l / theta : l * theta;
        if (n) l = l - freq * static_cast<float>(n) - pres;
        return v != 0.f ? l + v : l;
    };

    const int n0 = P.node_begin + blockIdx.z * P.rows_per_cta;
    const int n1 = min(n0 + P.rows_per_cta, P.node_end);
    auto mask_row = [&](int n) {                     // -1: none
        if (!P.masks || n >= n1) return -1LL;
        const long long item = static_cast<long long>(b) * P.n_nodes + n;
        return P.mask_index ? static_cast<long long>(__ldg(P.mask_index + item)) : item;
    };
    long long m_next = mask_row(n0 + warp);
    for (int n = n0 + warp; n < n1; n += kWarps) {
        const long long r = static_cast<long long>(b) * P.rows_per_tree + n;
        const char *src = static_cast<const char *>(P.logits) + (r * P.ld_in + x0) * T::kBytes;
        char *dst = static_cast<char *>(P.out) + (r * P.ld_out + x0) * T::kBytes;
        const uint32_t *mask = nullptr;
        const long long m = m_next;
        m_next = mask_row(n + kWarps);               // (in flight while this row is worked on)
        if (m >= 0 && m < P.n_masks) mask = P.masks + m * P.ld_mask + (x0 >> 5);
        else if (m >= 0 && P.status && blockIdx.x == 0 && lane == 0) atomicOr(&P.status[b], MCSD_STATUS_BAD_MASK);
        auto allowed = [&](int i) { return !mask || ((__ldg(mask + (i >> 5)) >> (i & 31)) & 1u); };
        auto mask_one = [&](int i) {
            if (!allowed(i)) store_elem<DT>(dst, i, -INFINITY);
            else if (!P.in_place) store_elem<DT>(dst, i, load_elem<DT>(src, i));
        };
        // the path: lane i the i-th ancestor, root excluded
        int length = 0;
        if (penalise && P.cand) {
            for (int i0 = 0; i0 < P.depth; i0 += 32) {
                int a = n;
                for (int i = 0; i < i0 + lane && a > 0; ++i) a = P.parent[a];
                if (a > 0 && i0 + lane < P.depth) {
                    const uint32_t t = static_cast<uint32_t>(s_cand[a]) - static_cast<uint32_t>(x0);
                    const bool here = t < static_cast<uint32_t>(n_el);
                    s_token[i0 + lane] = here ? static_cast<int32_t>(t) : -1;
                    if (here) s_value[i0 + lane] = load_elem<DT>(src, t);
                }
                length += __popc(__ballot_sync(0xffffffffu, a > 0 && i0 + lane < P.depth));
            }
        }
        // the first of the listed tokens' logits are asked for now, so that they arrive with the row's
        constexpr int kAhead = 2;
        float ahead[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) ahead[k] = lane + 32 * k < listed ? load_elem<DT>(src, s_list[lane + 32 * k]) : 0.f;
        __syncwarp();                                // read before any lane writes the row in place
        // the mask alone; in place only what it takes out is written
        if constexpr (VEC) {
            const int n_vec = n_el / VE;
            // the slice's words of the mask, word lane + 32 j with this lane
            constexpr int kWords = kRulesMaxSlice / 1024;
            uint32_t words[kWords];
#pragma unroll
            for (int j = 0; j < kWords; ++j) words[j] = mask && 32 * (lane + 32 * j) < n_el ? __ldg(mask + lane + 32 * j) : 0xffffffffu;
            if (!P.in_place || mask)
#pragma unroll
                for (int pass = 0; pass < kRulesMaxSlice / (32 * kFlight * VE); ++pass) {
                    const int v0 = lane + pass * 32 * kFlight;
                    if (pass * 32 * kFlight >= n_vec) break;
                    uint4 v[kFlight];
                    uint32_t keep[kFlight];
#pragma unroll
                    for (int k = 0; k < kFlight; ++k) {
                        const int i = (v0 + 32 * k) * VE;
                        const bool in = v0 + 32 * k < n_vec;
                        if (!P.in_place) v[k] = ld_plain_v4_if(src + static_cast<long long>(i) * T::kBytes, in);
                        // (word i / 32: 32 / VE lanes share one, a vector further on lies VE words on)
                        const int word = pass * kFlight * VE + k * VE + lane / (32 / VE);
                        const uint32_t bits = __shfl_sync(0xffffffffu, words[(pass * kFlight + k) * VE / 32], word & 31) >> (i & 31);
                        keep[k] = in ? bits & kAll : kAll;
                    }
                    if (P.in_place) {
#pragma unroll
                        for (int k = 0; k < kFlight; ++k)
                            v[k] = ld_plain_v4_if(src + static_cast<long long>(v0 + 32 * k) * 16, keep[k] != 0u && keep[k] != kAll);
                    }
#pragma unroll
                    for (int k = 0; k < kFlight; ++k) {
                        if (v0 + 32 * k >= n_vec || (P.in_place && keep[k] == kAll)) continue;
                        uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t m;
                            if constexpr (VE == 4) m = 0u - ((keep[k] >> j) & 1u);
                            else m = ((keep[k] >> (2 * j)) & 1u) * 0xffffu | ((keep[k] >> (2 * j + 1)) & 1u) * 0xffff0000u;
                            w[j] = (w[j] & m) | (T::kNegInfWord & ~m);
                        }
                        reinterpret_cast<uint4 *>(dst)[v0 + 32 * k] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            const int i = n_vec * VE + lane;         // the last tokens of the vocabulary, one by one
            if (i < n_el) mask_one(i);
        } else if (!P.in_place || mask) {
            for (int i = lane; i < n_el; i += 32) mask_one(i);
        }
        __syncwarp();
        // the tokens some rule concerns
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (lane + 32 * k < listed) {
                const int i = s_list[lane + 32 * k];
                if (allowed(i)) store_elem<DT>(dst, i, apply(ahead[k], s_count[i], s_bias[i]));
            }
        for (int k = lane + 32 * kAhead; k < listed; k += 32) {
            const int i = s_list[k];
            if (allowed(i)) store_elem<DT>(dst, i, apply(load_elem<DT>(src, i), s_count[i], s_bias[i]));
        }
        __syncwarp();
        // the tokens of the path: the first of equal ones writes, with all of them counted
        for (int i = lane; i < length; i += 32) {
            const int t = s_token[i];
            if (t < 0 || !allowed(t)) continue;
            uint32_t more = 0;
            bool head = true;
            for (int j = 0; j < length; ++j)
                if (s_token[j] == t) {
                    ++more;
                    head = head && j >= i;
                }
            if (head) store_elem<DT>(dst, t, apply(s_value[i], s_count[t] + more, s_bias[t]));
        }
        __syncwarp();
    }
}

}  // namespace mcsd
