// Log probabilities of given tokens, entropy and the largest tokens of rows of logits.
#pragma once

#include "mcsd_common.cuh"

namespace mcsd {

constexpr int kLogprobThreads = 256;

struct LogprobParams {
    const void *logits;
    long long ld, n_logits, n_out;
    const int32_t *row_index, *path_nodes, *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *top_ids;
    int32_t V, n_given, n_top, path_len, nodes_per_tree;
    float inv_t;
};

// Row of the logits that output row i reads, -1 if none.
__device__ __forceinline__ long long logprob_row(const LogprobParams &P, long long i)
{
    long long r = i;
    if (P.path_nodes) {
        const long long b = i / P.path_len, j = i - b * P.path_len;
        const int node = j == 0 ? 0 : P.path_nodes[i - 1];
        if (node < 0 || node >= P.nodes_per_tree) return -1;
        r = b * P.nodes_per_tree + node;
    } else if (P.row_index) {
        r = P.row_index[i];
    }
    return r < 0 || r >= P.n_logits ? -1 : r;
}

// Logits as whole numbers in their order (both zeros alike), behind them the token, lower ones first.
__device__ __forceinline__ unsigned long long logit_key(float l, int x)
{
    const uint32_t u = __float_as_uint(l + 0.f);
    const uint32_t order = (u >> 31) ? ~u : u | 0x80000000u;
    return static_cast<unsigned long long>(order) << 32 | static_cast<uint32_t>(~x);
}

template <int DT>
__global__ void __launch_bounds__(kLogprobThreads)
logprob_kernel(const __grid_constant__ LogprobParams P)
{
    __shared__ unsigned long long s_key[kLogprobThreads / 32];
    __shared__ double s_sum[2][kLogprobThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (long long i = blockIdx.x; i < P.n_out; i += gridDim.x) {
        const long long r = logprob_row(P, i);
        if (r < 0) continue;
        const char *row = static_cast<const char *>(P.logits) + r * P.ld * Elem<DT>::kBytes;
        float m = -INFINITY;
        bool bad = false;
        for (int x = tid; x < P.V; x += kLogprobThreads) {
            const float l = Elem<DT>::load(row, x);
            bad |= !(l < INFINITY);
            m = fmaxf(m, l);
        }
        m = warp_max(m);
        bad = __syncthreads_or(bad);
        if (lane == 0) s_sum[0][warp] = m;
        __syncthreads();
        for (int w = 0; w < kLogprobThreads / 32; ++w) m = fmaxf(m, static_cast<float>(s_sum[0][w]));
        __syncthreads();
        double z = 0.0, e = 0.0;
        if (m > -INFINITY && !bad)
            for (int x = tid; x < P.V; x += kLogprobThreads) {
                const float l = Elem<DT>::load(row, x);
                const float d = (l - m) * P.inv_t, p = expf(d);
                z += p;
                if (p > 0.f) e += static_cast<double>(p) * d;
            }
        for (int o = 16; o > 0; o >>= 1) { z += __shfl_xor_sync(0xffffffffu, z, o); e += __shfl_xor_sync(0xffffffffu, e, o); }
        if (lane == 0) { s_sum[0][warp] = z; s_sum[1][warp] = e; }
        __syncthreads();
        z = e = 0.0;
        for (int w = 0; w < kLogprobThreads / 32; ++w) { z += s_sum[0][w]; e += s_sum[1][w]; }
        const float none = __int_as_float(0x7fc00000), log_z = m > -INFINITY && !bad ? static_cast<float>(log(z)) : none;
        if (tid == 0 && P.entropy) P.entropy[i] = log_z - static_cast<float>(e / z);
        if (P.logprobs)
            for (int g = tid; g < P.n_given; g += kLogprobThreads) {
                const int x = P.tokens[i * P.n_given + g];
                P.logprobs[i * P.n_given + g] = x < 0 || x >= P.V ? none : (Elem<DT>::load(row, x) - m) * P.inv_t - log_z;
            }
        unsigned long long last = ~0ull;
        for (int k = 0; k < P.n_top; ++k) {
            unsigned long long best = 0ull;
            for (int x = tid; x < P.V; x += kLogprobThreads) {
                const unsigned long long key = logit_key(Elem<DT>::load(row, x), x);
                if (key < last && key > best) best = key;
            }
            for (int o = 16; o > 0; o >>= 1) { const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o); best = best > other ? best : other; }
            if (lane == 0) s_key[warp] = best;
            __syncthreads();
            for (int w = 0; w < kLogprobThreads / 32; ++w) best = best > s_key[w] ? best : s_key[w];
            __syncthreads();
            const int x = static_cast<int>(~static_cast<uint32_t>(best));
            if (tid == 0) {
                const bool there = m > -INFINITY && !bad;
                if (P.top_ids) P.top_ids[i * P.n_top + k] = there ? x : -1;
                if (P.top_logprobs) P.top_logprobs[i * P.n_top + k] = there ? (Elem<DT>::load(row, x) - m) * P.inv_t - log_z : none;
            }
            last = best;
        }
        __syncthreads();
    }
}

}  // namespace mcsd
