// Eviction of cached rows by gathered weight: each key/value head of each layer keeps the heaviest of its own.
#pragma once

#include "mcsd_cache.cuh"

namespace mcsd {

constexpr int kEvictThreads = 256;
constexpr int kEvictKeys = 8192;                    // weights that are kept on chip between the passes over them

struct EvictParams {
    CacheParams c;
    long long n_layers, layer_stride, weight_stride, ld_table;
    const int32_t *table, *len, *keep_len;
    float *weights;
    int32_t *len_out;
    int32_t batch, max_pages, keep, sink, recent;
    int32_t n_keys;                                 // room for weights in shared memory
};

// Weights as whole numbers in their order (both zeros alike), a NaN below all.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);    // (-0 becomes 0)
    return w != w ? 0u : (u >> 31) ? ~u : u | 0x80000000u;
}

// One CTA per (layer, sequence, head) at a time. The bar, the largest weight that enough rows reach, comes from four passes over the
// weights, eight bits each (a count of every value of the bits in shared memory, then a search from the top); up to kEvictKeys
// weights stay in shared memory between the passes. Then the rows are gone through in order, 256 at a time: those
// that stay get their places by ballots and are moved, 16 bytes a thread, all of a round read before one is written. A place is never behind
// its row, so that a round overwrites nothing that a later one reads, and the next round's places are found while rows are on their way.
template <int D>
__global__ void __launch_bounds__(kEvictThreads, 4)
evict_kernel(const __grid_constant__ EvictParams P)
{
    constexpr int WARPS = kEvictThreads / 32, CH = D / 16;          // 16-byte pieces of a row: keys, then values
    extern __shared__ uint32_t s_key[];
    __shared__ int s_count[WARPS], s_tie[WARPS], s_bins[256], s_pick[2];
    __shared__ int s_from[kEvictThreads], s_from_page[kEvictThreads], s_to[kEvictThreads], s_to_page[kEvictThreads];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = 1 << P.c.page_shift;
    const long long items = P.n_layers * P.batch * P.c.n_heads;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int head = static_cast<int>(item % P.c.n_heads), b = static_cast<int>(item / P.c.n_heads % P.batch);
        const long long layer = item / P.c.n_heads / P.batch;
        const int held = __ldg(P.len + b), keep = P.keep_len ? __ldg(P.keep_len + b) : P.keep;
        const int len = static_cast<int>(min(static_cast<long long>(held), static_cast<long long>(P.max_pages) << P.c.page_shift));
        const bool cut = held >= 0 && keep >= 0 && len > keep;
        if (layer == 0 && head == 0 && tid == 0 && P.len_out) P.len_out[b] = cut ? keep : held;
        if (!cut) continue;
        const int sink = min(P.sink, keep), recent = min(P.recent, keep - sink), want = keep - sink - recent, end = len - recent;
        const int32_t *table = P.table + b * P.ld_table;
        float *weights = P.weights + layer * P.weight_stride;
        unsigned char *pages = P.c.pages + layer * P.layer_stride + static_cast<long long>(head) * kv_block_bytes(D, ps);
        auto page_of = [&](int pos) {
            const int page = __ldg(table + (pos >> P.c.page_shift));
            return page < 0 || page >= P.c.n_pages ? -1 : page;
        };
        auto weight_at = [&](int page, int pos) -> float * { return weights + (static_cast<long long>(page) * P.c.n_heads + head) * ps + (pos & (ps - 1)); };
        auto read_key = [&](int pos) {
            const int page = page_of(pos);
            return page < 0 ? 0u : weight_key(*weight_at(page, pos));
        };
        // ---- the bar: `want` of the keys of [sink, end) are above it, or equal to it and among the first `ties` that are
        const int n = end - sink, held_keys = min(n, P.n_keys);
        for (int i = tid; i < held_keys; i += kEvictThreads) s_key[i] = read_key(sink + i);
        auto key_of = [&](int i) { return i < held_keys ? s_key[i] : read_key(sink + i); };
        uint32_t bar = 0u;
        int ties = want;
        if (want == 0) {
            bar = 0xffffffffu;                      // (the key of no number)
        } else {
            for (int shift = 24; shift >= 0; shift -= 8) {
                s_bins[tid] = 0;
                __syncthreads();                    // (for the first pass: the keys are there, too)
                for (int i = tid; i < n; i += kEvictThreads) {
                    const uint32_t key = key_of(i);
                    if (shift == 24 || (key ^ bar) >> (shift + 8) == 0u) atomicAdd(&s_bins[key >> shift & 255u], 1);
                }
                __syncthreads();
                // keys in bins above this thread's
                const int bin = 255 - tid, own = s_bins[bin];
                int above = own;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, above, o);
                    if (lane >= o) above += up;
                }
                if (lane == 31) s_count[warp] = above;
                __syncthreads();
                for (int w = 0; w < warp; ++w) above += s_count[w];
                above -= own;
                if (above < ties && above + own >= ties) { s_pick[0] = bin; s_pick[1] = ties - above; }
                __syncthreads();
                bar |= static_cast<uint32_t>(s_pick[0]) << shift;
                ties = s_pick[1];
            }
        }
        // ---- the rows, 256 at a time
        int kept = sink;
        for (int pos0 = sink; pos0 < len; pos0 += kEvictThreads) {
            const int pos = pos0 + tid;
            const uint32_t key = pos < end ? key_of(pos - sink) : 0u;
            const bool safe = pos >= end && pos < len, tie = pos < end && key == bar;
            const unsigned tie_mask = __ballot_sync(0xffffffffu, tie);
            if (lane == 0) s_tie[warp] = __popc(tie_mask);
            __syncthreads();                        // (and the round before has read its places)
            int before = __popc(tie_mask & ((1u << lane) - 1u)), all = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) { before += w < warp ? s_tie[w] : 0; all += s_tie[w]; }
            const bool stays = safe || (pos < end && key > bar) || (tie && before < ties);
            ties -= min(all, ties);
            const unsigned mask = __ballot_sync(0xffffffffu, stays);
            if (lane == 0) s_count[warp] = __popc(mask);
            __syncthreads();
            int rank = __popc(mask & ((1u << lane) - 1u)), count = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) { rank += w < warp ? s_count[w] : 0; count += s_count[w]; }
            if (stays) {
                const int to = kept + rank, from_page = page_of(pos), to_page = page_of(to);
                const bool moves = to != pos && from_page >= 0 && to_page >= 0;
                s_from[rank] = pos;
                s_to[rank] = to;
                s_from_page[rank] = moves ? from_page : -1;
                s_to_page[rank] = to_page;
            }
            kept += count;
            __syncthreads();
            uint4 row[CH];
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                const int x = tid + u * kEvictThreads, j = x / CH, c = x % CH;
                if (j < count && s_from_page[j] >= 0)
                    row[u] = *reinterpret_cast<const uint4 *>(pages + s_from_page[j] * P.c.page_stride + ((c / (CH / 2)) * ps + (s_from[j] & (ps - 1))) * (D / 2) + (c % (CH / 2)) * 16);
            }
            uint32_t key_param = 0u, value_param = 0u;
            float weight = 0.f;
            const bool mine = tid < count && s_from_page[tid] >= 0;
            if (mine) {
                const uint32_t *param = reinterpret_cast<const uint32_t *>(pages + s_from_page[tid] * P.c.page_stride + ps * D) + (s_from[tid] & (ps - 1));
                key_param = param[0];
                value_param = param[ps];
                weight = *weight_at(s_from_page[tid], s_from[tid]);
            }
            __syncthreads();                        // every row of the round is read before one is written
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                const int x = tid + u * kEvictThreads, j = x / CH, c = x % CH;
                if (j < count && s_from_page[j] >= 0)
                    *reinterpret_cast<uint4 *>(pages + s_to_page[j] * P.c.page_stride + ((c / (CH / 2)) * ps + (s_to[j] & (ps - 1))) * (D / 2) + (c % (CH / 2)) * 16) = row[u];
            }
            if (mine) {
                uint32_t *param = reinterpret_cast<uint32_t *>(pages + s_to_page[tid] * P.c.page_stride + ps * D) + (s_to[tid] & (ps - 1));
                param[0] = key_param;
                param[ps] = value_param;
                *weight_at(s_to_page[tid], s_to[tid]) = weight;
            }
        }
        __syncthreads();
    }
}

}  // namespace mcsd
