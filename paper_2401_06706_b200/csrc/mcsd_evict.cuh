// Eviction of cached rows by gathered weight: each key/value head of each layer keeps the heaviest of its own.
#pragma once

#include "mcsd_cache.cuh"

namespace mcsd {

constexpr int kEvictThreads = 256;
constexpr int kEvictBins = 2048;                    // values of the eleven bits that a pass counts
constexpr int kEvictKeys = 7168;                    // weights that are kept on chip between the passes over them (with the bins, what a CTA has without asking)
constexpr int kEvictList = 4 * kEvictThreads;       // rows that are listed and not moved yet: a batch, the next one, and what a round adds

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

// One CTA per (layer, sequence, head) at a time. The bar, the largest weight that enough rows reach, comes from three passes over the
// weights, eleven bits each (a count of every value of the bits in shared memory, then a search from the top); up to kEvictKeys
// weights stay in shared memory between the passes. Then the rows are gone through in order: those that
// stay are listed by ballots and moved 256 at a time, 16 bytes a thread, all of a batch read before one is written. A place is never behind
// its row, so that a batch overwrites nothing that a later one reads; the next batch is listed while rows are on their way.
// Bound by the moves and what precedes them: with passes of eight bits, of a CTA's 92000 cycles 13000 went into reading the weights, 14000 into the passes,
// 65000 into moves of 64-byte rows (D = 128; keys, values, parameters), at about 5.5 TB/s while they last. 8 sequences, 32 layers, 8 heads of 128: 220 us, 93 for the bytes. Three
// passes of eleven bits instead of four of eight, and a CTA for each (layer, sequence, head) instead of a loop over them: 241 -> 220; four CTAs of
// 256 threads an SM, so that one's passes overlap another's moves; rows moved 256 at a time instead of one by one: 600 -> 254.
template <int D>
__global__ void __launch_bounds__(kEvictThreads, 4)
evict_kernel(const __grid_constant__ EvictParams P)
{
    constexpr int WARPS = kEvictThreads / 32, CH = D / 16;          // 16-byte pieces of a row: keys, then values
    extern __shared__ uint32_t s_key[];
    __shared__ int s_count[WARPS], s_tie[WARPS], s_pick[2];
    __shared__ __align__(16) int s_bins[kEvictBins];
    __shared__ int s_from[kEvictList];              // rows that stay, a ring
    __shared__ longlong2 s_move[kEvictThreads];     // of a batch: offsets of the key codes where a row is and where it goes, -1: it stays where it is
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = 1 << P.c.page_shift;
    const long long items = P.n_layers * P.batch * P.c.n_heads;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {      // (one, but for a million CTAs)
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
        for (int i0 = tid; i0 < held_keys; i0 += 8 * kEvictThreads) {           // (eight pages, then eight weights on their way)
            int page[8];
            float w[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) page[u] = i0 + u * kEvictThreads < held_keys ? page_of(sink + i0 + u * kEvictThreads) : -1;
#pragma unroll
            for (int u = 0; u < 8; ++u) w[u] = page[u] < 0 ? 0.f : *weight_at(page[u], sink + i0 + u * kEvictThreads);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i0 + u * kEvictThreads < held_keys) s_key[i0 + u * kEvictThreads] = page[u] < 0 ? 0u : weight_key(w[u]);
        }
        auto key_of = [&](int i) { return i < held_keys ? s_key[i] : read_key(sink + i); };
        uint32_t bar = 0u;
        int ties = want;
        if (want == 0) {
            bar = 0xffffffffu;                      // (the key of no number)
        } else {
            for (int shift = 21; shift >= 0; shift = shift == 10 ? 0 : shift - 11) {        // bits 31..21, 20..10, 9..0
                const int bits = shift == 0 ? 10 : 11;
#pragma unroll
                for (int u = 0; u < kEvictBins / 4 / kEvictThreads; ++u) reinterpret_cast<int4 *>(s_bins)[tid + u * kEvictThreads] = make_int4(0, 0, 0, 0);
                __syncthreads();                    // (for the first pass: the keys are there, too)
                for (int i = tid; i < n; i += kEvictThreads) {
                    const uint32_t key = key_of(i);
                    if (shift == 21 || (key ^ bar) >> (shift + bits) == 0u) atomicAdd(&s_bins[key >> shift & ((1u << bits) - 1u)], 1);
                }
                __syncthreads();
                // each thread has eight bins, the highest first; how many keys are above them
                const int top = kEvictBins - 1 - 8 * tid;
                int own[8], sum = 0;
#pragma unroll
                for (int u = 0; u < 8; ++u) { own[u] = s_bins[top - u]; sum += own[u]; }
                int above = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, above, o);
                    if (lane >= o) above += up;
                }
                if (lane == 31) s_count[warp] = above;
                __syncthreads();
                for (int w = 0; w < warp; ++w) above += s_count[w];
                above -= sum;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    if (above < ties && above + own[u] >= ties) { s_pick[0] = top - u; s_pick[1] = ties - above; }
                    above += own[u];
                }
                __syncthreads();
                bar |= static_cast<uint32_t>(s_pick[0]) << shift;
                ties = s_pick[1];
            }
        }
        // ---- the rows in order: those that stay are listed, and moved 256 at a time
        int listed = 0, moved = 0, pos0 = sink;     // rows listed and moved so far; the next position to look at
        // Goes on until `upto` rows are listed or there are no more.
        auto list = [&](int upto) {
            while (pos0 < len && listed < upto) {
                const int pos = pos0 + tid;
                pos0 += kEvictThreads;
                const uint32_t key = pos < end ? key_of(pos - sink) : 0u;
                const bool safe = pos >= end && pos < len, tie = pos < end && key == bar;
                const unsigned tie_mask = __ballot_sync(0xffffffffu, tie), sure = __ballot_sync(0xffffffffu, safe || (pos < end && key > bar));
                __syncthreads();                    // (the counts of the round before are read)
                if (lane == 0) { s_tie[warp] = __popc(tie_mask); s_count[warp] = __popc(sure); }
                __syncthreads();
                // (a warp's ties are kept as far as those of the warps before it leave room)
                int left = ties, rank = listed, all = 0, room = 0;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) {
                    const int took = min(s_tie[w], left);
                    if (w < warp) rank += s_count[w] + took;
                    if (w == warp) room = took;
                    all += s_count[w] + took;
                    left -= took;
                }
                ties = left;
                const bool stays = safe || (pos < end && key > bar) || (tie && __popc(tie_mask & ((1u << lane) - 1u)) < room);
                const unsigned mask = __ballot_sync(0xffffffffu, stays);
                if (stays) s_from[(rank + __popc(mask & ((1u << lane) - 1u))) % kEvictList] = pos;
                listed += all;
            }
            __syncthreads();
        };
        list(kEvictThreads);
        while (moved < listed) {
            const int count = min(listed - moved, kEvictThreads);
            // where this thread's row comes from and goes to
            int from = 0, to = 0, from_page = -1, to_page = -1;
            if (tid < count) {
                from = s_from[(moved + tid) % kEvictList];
                to = sink + moved + tid;
                if (from != to) {
                    from_page = page_of(from);
                    to_page = page_of(to);
                    if (to_page < 0) from_page = -1;
                }
                s_move[tid] = from_page < 0 ? make_longlong2(-1, 0) :
                    make_longlong2(from_page * P.c.page_stride + (from & (ps - 1)) * (D / 2), to_page * P.c.page_stride + (to & (ps - 1)) * (D / 2));
            }
            __syncthreads();
            uint4 row[CH];
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                const int x = tid + u * kEvictThreads, j = x / CH, c = x % CH;
                if (j < count && s_move[j].x >= 0)
                    row[u] = *reinterpret_cast<const uint4 *>(pages + s_move[j].x + (c / (CH / 2)) * ps * (D / 2) + (c % (CH / 2)) * 16);
            }
            uint32_t key_param = 0u, value_param = 0u;
            float weight = 0.f;
            if (from_page >= 0) {
                const uint32_t *param = reinterpret_cast<const uint32_t *>(pages + from_page * P.c.page_stride + ps * D) + (from & (ps - 1));
                key_param = param[0];
                value_param = param[ps];
                weight = *weight_at(from_page, from);
            }
            list(moved + 2 * kEvictThreads);        // (the next batch, while these rows are on their way; its barriers stand between reading and writing)
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                const int x = tid + u * kEvictThreads, j = x / CH, c = x % CH;
                if (j < count && s_move[j].x >= 0)
                    *reinterpret_cast<uint4 *>(pages + s_move[j].y + (c / (CH / 2)) * ps * (D / 2) + (c % (CH / 2)) * 16) = row[u];
            }
            if (from_page >= 0) {
                uint32_t *param = reinterpret_cast<uint32_t *>(pages + to_page * P.c.page_stride + ps * D) + (to & (ps - 1));
                param[0] = key_param;
                param[ps] = value_param;
                *weight_at(to_page, to) = weight;
            }
            moved += count;
            __syncthreads();                        // (the places of these rows are read)
        }
        __syncthreads();
    }
}

}  // namespace mcsd
