// Eviction of cached rows by gathered weight: each key/value head of each layer keeps the heaviest of its own.
#pragma once

#include "mcsd_cache.cuh"

namespace mcsd {

constexpr int kEvictThreads = 256;

struct EvictParams {
    CacheParams c;
    long long n_layers, layer_stride, weight_stride, ld_table;
    const int32_t *table, *len, *keep_len;
    float *weights;
    int32_t *len_out;
    int32_t batch, max_pages, keep, sink, recent;
};

// Weights as whole numbers in their order (both zeros alike), a NaN below all.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);    // (-0 becomes 0)
    return w != w ? 0u : (u >> 31) ? ~u : u | 0x80000000u;
}

// A CTA per (layer, sequence, head).
template <int D>
__global__ void __launch_bounds__(kEvictThreads)
evict_kernel(const __grid_constant__ EvictParams P)
{
    __shared__ int s_count[kEvictThreads / 32], s_tie[kEvictThreads / 32], s_from[kEvictThreads], s_to[kEvictThreads];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = 1 << P.c.page_shift;
    const long long items = P.n_layers * P.batch * P.c.n_heads;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int head = static_cast<int>(item % P.c.n_heads), b = static_cast<int>(item / P.c.n_heads % P.batch);
        const long long layer = item / P.c.n_heads / P.batch;
        const int held = P.len[b], keep = P.keep_len ? P.keep_len[b] : P.keep;
        const int len = static_cast<int>(min(static_cast<long long>(held), static_cast<long long>(P.max_pages) << P.c.page_shift));
        const bool cut = held >= 0 && keep >= 0 && len > keep;
        if (layer == 0 && head == 0 && tid == 0 && P.len_out) P.len_out[b] = cut ? keep : held;
        if (!cut) continue;
        const int sink = min(P.sink, keep), recent = min(P.recent, keep - sink), want = keep - sink - recent;
        const int32_t *table = P.table + b * P.ld_table;
        float *weights = P.weights + layer * P.weight_stride;
        unsigned char *pages = P.c.pages + layer * P.layer_stride + static_cast<long long>(head) * kv_block_bytes(D, ps);
        auto page_of = [&](int pos) {
            const int page = table[pos >> P.c.page_shift];
            return page < 0 || page >= P.c.n_pages ? -1 : page;
        };
        auto weight_of = [&](int pos) -> float * {
            const int page = page_of(pos);
            return page < 0 ? nullptr : weights + (static_cast<long long>(page) * P.c.n_heads + head) * ps + (pos & (ps - 1));
        };
        auto key_of = [&](int pos) { const float *w = weight_of(pos); return w ? weight_key(*w) : 0u; };
        auto block_sum = [&](int v) {
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            __syncthreads();
            if (lane == 0) s_count[warp] = v;
            __syncthreads();
            int sum = 0;
            for (int w = 0; w < kEvictThreads / 32; ++w) sum += s_count[w];
            return sum;
        };
        // the largest threshold with at least `want` keys at or above it, bit by bit; `ties`: how many of those equal to it are kept
        uint32_t bar = 0u;
        int ties = want;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t higher = bar | 1u << bit;
            int n = 0;
            for (int pos = sink + tid; pos < len - recent; pos += kEvictThreads) n += key_of(pos) >= higher;
            if (block_sum(n) >= want) bar = higher;
        }
        {
            int n = 0;
            for (int pos = sink + tid; pos < len - recent; pos += kEvictThreads) n += key_of(pos) > bar;
            ties = want - block_sum(n);
        }
        int kept = sink;
        for (int pos0 = sink; pos0 < len; pos0 += kEvictThreads) {
            const int pos = pos0 + tid;
            const uint32_t key = pos < len - recent ? key_of(pos) : 0u;
            const bool safe = pos >= len - recent && pos < len, tie = pos < len - recent && key == bar;
            const unsigned tie_mask = __ballot_sync(0xffffffffu, tie);
            __syncthreads();
            if (lane == 0) s_tie[warp] = __popc(tie_mask);
            __syncthreads();
            int before = __popc(tie_mask & ((1u << lane) - 1u)), all = 0;
            for (int w = 0; w < kEvictThreads / 32; ++w) { before += w < warp ? s_tie[w] : 0; all += s_tie[w]; }
            const bool stays = safe || (pos < len - recent && key > bar) || (tie && before < ties);
            ties -= min(all, ties);
            const unsigned mask = __ballot_sync(0xffffffffu, stays);
            if (lane == 0) s_count[warp] = __popc(mask);
            __syncthreads();
            int rank = __popc(mask & ((1u << lane) - 1u)), n = 0;
            for (int w = 0; w < kEvictThreads / 32; ++w) { rank += w < warp ? s_count[w] : 0; n += s_count[w]; }
            if (stays) { s_from[rank] = pos; s_to[rank] = kept + rank; }
            __syncthreads();
            // the rows of this round, one thread a row: read, then (when all are read) written
            unsigned char *to = nullptr;
            uint4 row[D / 16];
            uint32_t key_param = 0u, value_param = 0u;
            float w = 0.f, *w_to = nullptr;
            int to_row = 0;
            if (tid < n && s_from[tid] != s_to[tid] && page_of(s_from[tid]) >= 0 && page_of(s_to[tid]) >= 0) {
                const int from_row = s_from[tid] & (ps - 1);
                const unsigned char *from = pages + page_of(s_from[tid]) * P.c.page_stride;
                to = pages + page_of(s_to[tid]) * P.c.page_stride;
                to_row = s_to[tid] & (ps - 1);
                for (int i = 0; i < D / 32; ++i) {
                    row[i] = *reinterpret_cast<const uint4 *>(from + from_row * (D / 2) + 16 * i);
                    row[D / 32 + i] = *reinterpret_cast<const uint4 *>(from + (ps + from_row) * (D / 2) + 16 * i);
                }
                key_param = *reinterpret_cast<const uint32_t *>(from + ps * D + 4 * from_row);
                value_param = *reinterpret_cast<const uint32_t *>(from + ps * D + 4 * (ps + from_row));
                w = *weight_of(s_from[tid]);
                w_to = weight_of(s_to[tid]);
            }
            __syncthreads();
            if (to) {
                for (int i = 0; i < D / 32; ++i) {
                    *reinterpret_cast<uint4 *>(to + to_row * (D / 2) + 16 * i) = row[i];
                    *reinterpret_cast<uint4 *>(to + (ps + to_row) * (D / 2) + 16 * i) = row[D / 32 + i];
                }
                *reinterpret_cast<uint32_t *>(to + ps * D + 4 * to_row) = key_param;
                *reinterpret_cast<uint32_t *>(to + ps * D + 4 * (ps + to_row)) = value_param;
                *w_to = w;
            }
            kept += n;
        }
        __syncthreads();
    }
}

}  // namespace mcsd
