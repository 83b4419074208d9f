// pages_kernel: page tables and slot maps of a paged key/value cache, from the lengths of the requests.
#pragma once

#include "mcsd_common.cuh"

namespace mcsd {

constexpr int kPagesThreads = 1024;

struct PagesParams {
    const int32_t *start, *count;
    int32_t *table;
    int32_t *held, *held_out;
    int32_t *ring, *state, *state_out;
    long long *slots;
    int32_t *cu_tokens, *status;
    long long ld_table, n_slots;
    int32_t batch, page_shift, max_pages, new_tokens, cap, commit_last;
};

// Exclusive sums over the CTA's threads of three values; `total` gets the sums (all threads).
__device__ __forceinline__ void pages_scan(long long (&v)[3], long long (&total)[3], long long (*s_warp)[3], int tid)
{
    const int lane = tid & 31, warp = tid >> 5;
    long long incl[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        incl[q] = v[q];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, incl[q], o);
            if (lane >= o) incl[q] += t;
        }
        if (lane == 31) s_warp[warp][q] = incl[q];
    }
    __syncthreads();
    long long off[3] = {0, 0, 0};
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        // every warp sums the warp totals for itself
        const long long t = s_warp[lane][q];
        long long inc = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        off[q] = __shfl_sync(0xffffffffu, inc - t, warp);
        total[q] = __shfl_sync(0xffffffffu, inc, 31);
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) v[q] = off[q] + incl[q] - v[q];
    __syncthreads();
}

// Every CTA forms the prefix sums over all sequences for itself (at most MCSD_MAX_SEQUENCES, a few
// passes of one block-wide scan) and keeps them in shared memory; then the table entries and the
// slots are spread over the whole grid.  A slot's page is taken from where the table entry comes from
// (the old entry, or the ring), so nothing waits for another CTA's writes: one launch.  The ring lets
// the pages taken and the pages returned lie in different places, so reads and writes of a call never
// meet.  New lengths and the new state are written by CTA 0, or, where they replace their inputs, by
// the CTA that finishes last (counted in state[2], which goes back to 0).  Bound by latency: three dependent
// loads and two block-wide scans; a call takes 10 us for 8 sequences (of which only a
// warp's worth has anything to scan), 15 us for 256 prompts and 1.05 M slots.
__global__ void __launch_bounds__(kPagesThreads)
pages_kernel(const PagesParams P)
{
    __shared__ long long s_warp[32][3];
    __shared__ int s_last;
    extern __shared__ int32_t s_pages[];
    int32_t *s_tok = s_pages;                        // [batch + 1] first token of each sequence
    int32_t *s_take = s_tok + P.batch + 1;           // [batch] first ring entry taken, -1 - old pages if refused
    int32_t *s_give = s_take + P.batch;              // [batch] first ring entry returned
    int32_t *s_held = s_give + P.batch;              // [batch]
    int32_t *s_want = s_held + P.batch;              // [batch] pages held afterwards
    const int tid = threadIdx.x;
    const int ps_mask = (1 << P.page_shift) - 1;
    int head = P.state[0], n_free = P.state[1];
    head = head >= 0 && head < P.cap ? head : 0;
    n_free = min(max(n_free, 0), P.cap);

    long long run[3] = {0, 0, 0};                    // pages wanted from the ring, pages returned, tokens
    long long taken = 0;
    for (int b0 = 0; b0 < P.batch; b0 += kPagesThreads) {
        const int b = b0 + tid;
        long long v[3] = {0, 0, 0}, total[3];
        int held = 0, want = 0, tokens = 0;
        bool wide = false;
        if (b < P.batch) {
            const int start = P.start[b];
            held = min(max(P.held[b], 0), P.max_pages);
            want = held;
            if (start >= 0) {
                tokens = max(P.count ? P.count[b] : P.new_tokens, 0);
                const long long need = (static_cast<long long>(start) + tokens + ps_mask) >> P.page_shift;
                wide = need > P.max_pages;
                if (!wide) want = static_cast<int>(need);
            }
            v[0] = max(want - held, 0);
            v[1] = max(held - want, 0);
            v[2] = tokens;
        }
        const long long grow = v[0];
        pages_scan(v, total, s_warp, tid);
        if (b < P.batch) {
            const bool refused = wide || (grow > 0 && run[0] + v[0] + grow > n_free);
            if (refused) want = held;
            s_tok[b] = static_cast<int32_t>(run[2] + v[2]);
            s_take[b] = refused ? -1 : static_cast<int32_t>(run[0] + v[0] < n_free ? run[0] + v[0] : n_free);
            s_give[b] = static_cast<int32_t>(run[1] + v[1]);
            s_held[b] = held;
            s_want[b] = want;
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) run[q] += total[q];
    }
    if (tid == 0) s_tok[P.batch] = static_cast<int32_t>(run[2]);
    __syncthreads();
    // pages taken: up to the last sequence that was served (the demands before the first refusal)
    for (int b0 = 0; b0 < P.batch; b0 += kPagesThreads) {
        const int b = b0 + tid;
        long long t = 0;
        if (b < P.batch && s_want[b] > s_held[b]) t = static_cast<long long>(s_take[b]) + s_want[b] - s_held[b];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, o));
        if ((tid & 31) == 0) s_warp[tid >> 5][0] = t;
        __syncthreads();
        t = s_warp[tid & 31][0];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, o));
        taken = max(taken, t);
        __syncthreads();
    }
    const int returned = static_cast<int>(min(run[1], static_cast<long long>(P.cap - n_free)));

    // table entries: a warp per sequence
    const int lane = tid & 31;
    const int n_warps = gridDim.x * (kPagesThreads / 32);
    for (int b = blockIdx.x * (kPagesThreads / 32) + (tid >> 5); b < P.batch; b += n_warps) {
        int32_t *row = P.table + b * P.ld_table;
        const int held = s_held[b], want = s_want[b];
        for (int j = held + lane; j < want; j += 32) {
            const long long at = static_cast<long long>(head) + s_take[b] + (j - held);
            row[j] = P.ring[at % P.cap];
        }
        for (int j = want + lane; j < held; j += 32) {
            const int k = s_give[b] + (j - want);
            if (k < returned) P.ring[(static_cast<long long>(head) + n_free + k) % P.cap] = row[j];
        }
        if (P.status && lane == 0) P.status[b] = s_take[b] < 0 ? MCSD_STATUS_NO_PAGES : 0;
    }
    if (P.cu_tokens && blockIdx.x == 0)
        for (int b = tid; b <= P.batch; b += kPagesThreads) P.cu_tokens[b] = s_tok[b];
    if (P.slots) {
        // a warp per run of 256 tokens: one search for the run's first token, then steps to the next sequence
        const long long n = min(run[2], P.n_slots);
        for (long long t0 = 256ll * (blockIdx.x * (kPagesThreads / 32) + (tid >> 5)); t0 < n; t0 += 256ll * n_warps) {
            int lo = 0, hi = P.batch - 1;            // last sequence whose first token is <= t0
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_tok[mid] <= t0) lo = mid; else hi = mid - 1;
            }
            int b = lo;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const long long t = t0 + u * 32 + lane;
                if (t >= n) break;
                while (b + 1 < P.batch && s_tok[b + 1] <= t) ++b;
                long long slot = -1;
                if (s_take[b] >= 0) {
                    const int pos = P.start[b] + static_cast<int>(t - s_tok[b]);
                    const int j = pos >> P.page_shift;
                    // (out of the table only where the counts' sum passed 2^31, which has no packed order)
                    const bool there = j >= 0 && j < P.max_pages;
                    const int page = !there ? -1 : j < s_held[b] ? P.table[b * P.ld_table + j]
                                                                 : P.ring[(static_cast<long long>(head) + s_take[b] + (j - s_held[b])) % P.cap];
                    if (page >= 0) slot = (static_cast<long long>(page) << P.page_shift) + (pos & ps_mask);
                }
                P.slots[t] = slot;
            }
        }
    }
    bool commit = blockIdx.x == 0;
    if (P.commit_last && gridDim.x > 1) {
        __threadfence();
        __syncthreads();
        if (tid == 0) s_last = atomicAdd(&P.state[2], 1) == static_cast<int>(gridDim.x) - 1;
        __syncthreads();
        commit = s_last != 0;
    } else {
        __syncthreads();
    }
    if (commit) {
        for (int b = tid; b < P.batch; b += kPagesThreads) P.held_out[b] = s_want[b];
        if (tid == 0) {
            P.state_out[0] = static_cast<int32_t>((head + taken) % P.cap);
            P.state_out[1] = static_cast<int32_t>(n_free - taken + returned);
            if (P.commit_last) P.state[2] = 0;
        }
    }
}

}  // namespace mcsd
