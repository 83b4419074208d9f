// Attention of a flattened draft tree over the paged 4-bit cache.
#pragma once

#include "mcsd_cache.cuh"

namespace mcsd {

struct AttendParams {
    CacheParams c;
    const void *q;
    void *out;
    float *lse;                                     // may be null
    const int32_t *table, *prefix_len;
    long long ld_table;
    long long q_seq, q_node, q_head, o_seq, o_node, o_head;  // strides in elements
    int32_t batch, n_nodes, n_heads, max_pages;
    float scale;
    int16_t parent[MCSD_MAX_NODES];
};

// One warp per (sequence, node, query head): every lane owns D / 32 numbers of a row; keys are taken one
// after the other with a running maximum, sum and weighted sum in float32.
template <int DT, int D>
__global__ void __launch_bounds__(256)
attend_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    const long long row = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (row >= static_cast<long long>(P.batch) * P.n_nodes * P.n_heads) return;
    const int h = static_cast<int>(row % P.n_heads);
    const int n = static_cast<int>(row / P.n_heads % P.n_nodes);
    const int b = static_cast<int>(row / P.n_heads / P.n_nodes);
    const int prefix = P.prefix_len[b];
    if (prefix < 0) return;
    const int kv = h / (P.n_heads / P.c.n_heads), ps = 1 << P.c.page_shift;
    float q[E], acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] = load_elem<DT>(P.q, b * P.q_seq + n * P.q_node + h * P.q_head + lane * E + e);
        acc[e] = 0.f;
    }
    int node = n;
    for (long long i = 0;; ++i) {
        long long pos = i;
        if (i >= prefix) {                          // the prefix first, then the nodes up to the root
            if (node < 0) break;
            pos = static_cast<long long>(prefix) + node;
            node = P.parent[node];
        }
        const long long j = pos >> P.c.page_shift;
        if (j >= P.max_pages) continue;
        const int page = P.table[b * P.ld_table + j];
        if (page < 0 || page >= P.c.n_pages) continue;
        const int r = static_cast<int>(pos & (ps - 1));
        const unsigned char *block = P.c.pages + page * P.c.page_stride + static_cast<long long>(kv) * kv_block_bytes(D, ps);
        const __half2 *param = reinterpret_cast<const __half2 *>(block + ps * D) + r;
        const float2 kp = __half22float2(param[0]), vp = __half22float2(param[ps]);
        uint32_t kc = 0, vc = 0;
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
            kc |= block[r * (D / 2) + lane * (E / 2) + e] << (8 * e);
            vc |= block[(ps + r) * (D / 2) + lane * (E / 2) + e] << (8 * e);
        }
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) dot = fmaf(q[e], fmaf(kp.x, static_cast<float>((kc >> (4 * e)) & 15u) - 8.f, kp.y), dot);
        const float s = warp_sum(dot) * P.scale;
        const float top = fmaxf(m, s);
        const float keep = m == -INFINITY ? 0.f : expf(m - top), p = s == -INFINITY ? 0.f : expf(s - top);   // (a NaN score stays one)
        l = l * keep + p;
#pragma unroll
        for (int e = 0; e < E; ++e)
            acc[e] = acc[e] * keep + p * fmaf(vp.x, static_cast<float>((vc >> (4 * e)) & 15u) - 8.f, vp.y);
        m = top;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        store_elem<DT>(P.out, b * P.o_seq + n * P.o_node + h * P.o_head + lane * E + e, l > 0.f || !(l == l) ? acc[e] / l : 0.f);
    if (P.lse && lane == 0) P.lse[row] = l > 0.f || !(l == l) ? m + logf(l) : -INFINITY;
}

}  // namespace mcsd
