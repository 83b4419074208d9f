// Attention of a chunk of new tokens over the paged 4-bit cache, and the attention weight that its rows gather.
#pragma once

#include "mcsd_cache.cuh"

namespace mcsd {

struct ChunkParams {
    CacheParams c;
    const void *q;
    void *out;
    float *lse;                                     // of the attention: written (may be null); of the weights: read
    float *weights;
    const int32_t *table, *start, *cu;
    long long ld_table, n_tokens;
    long long q_token, q_head, o_token, o_head;     // strides in elements
    int32_t batch, n_heads, max_pages, max_new;
    int32_t group;                                  // query heads per key/value head
    int32_t last;                                   // tokens whose weights count, 0: all
    float scale, decay;
};

// The new tokens of sequence b: the row of the first one, how many, the positions there are before them and with them.
struct ChunkSeq { long long row; int count, start, len; };
template <typename P>
__device__ __forceinline__ ChunkSeq chunk_seq(const P &p, int b)
{
    ChunkSeq s;
    const int first = p.cu[b];
    long long n = static_cast<long long>(p.cu[b + 1]) - first;
    n = min(n, min(static_cast<long long>(p.max_new), p.n_tokens - first));
    s.start = p.start[b];
    s.row = first;
    s.count = s.start < 0 || first < 0 || n < 0 ? 0 : static_cast<int>(n);
    const long long there = static_cast<long long>(p.max_pages) << p.c.page_shift;
    s.len = static_cast<int>(min(static_cast<long long>(s.start) + s.count, there));
    return s;
}
// Positions that token i of the sequence sees.
__device__ __forceinline__ int chunk_sees(const ChunkSeq &s, int i) { return static_cast<int>(min(static_cast<long long>(s.start) + i + 1, static_cast<long long>(s.len))); }

// This lane's D / 32 numbers of the key (0) or value (1) row at `pos`; false if there is none.
template <int D>
__device__ __forceinline__ bool chunk_row(const CacheParams &c, const int32_t *table, int pos, int head, int which, int lane, float *x)
{
    const int page = table[pos >> c.page_shift];
    if (page < 0 || page >= c.n_pages) return false;
    unsigned char *codes;
    __half2 *param;
    kv_row<D>(c, (static_cast<long long>(page) << c.page_shift) + (pos & ((1 << c.page_shift) - 1)), head, which, codes, param);
    const float2 p = __half22float2(*param);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int d = lane * (D / 32) + i;
        x[i] = fmaf(p.x, static_cast<float>((codes[d >> 1] >> (4 * (d & 1))) & 15) - 8.f, p.y);
    }
    return true;
}

// A warp per (token, query head).
template <int DT, int D>
__global__ void __launch_bounds__(256)
chunk_kernel(const __grid_constant__ ChunkParams P)
{
    const int lane = threadIdx.x & 31, head = blockIdx.x;
    for (int b = blockIdx.y; b < P.batch; b += gridDim.y) {
        const ChunkSeq s = chunk_seq(P, b);
        const int32_t *table = P.table + b * P.ld_table;
        for (int i = blockIdx.z * 8 + (threadIdx.x >> 5); i < s.count; i += gridDim.z * 8) {
            float q[D / 32], o[D / 32], x[D / 32];
            const long long at = (s.row + i) * P.q_token + head * P.q_head + lane * (D / 32);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) { q[d] = load_elem<DT>(P.q, at + d); o[d] = 0.f; }
            float m = -INFINITY, l = 0.f;
            const int sees = chunk_sees(s, i);
            for (int pos = 0; pos < sees; ++pos) {
                if (!chunk_row<D>(P.c, table, pos, head / P.group, 0, lane, x)) continue;
                float z = 0.f;
#pragma unroll
                for (int d = 0; d < D / 32; ++d) z = fmaf(q[d], x[d], z);
                z = warp_sum(z) * P.scale;
                chunk_row<D>(P.c, table, pos, head / P.group, 1, lane, x);
                const float now = fmaxf(m, z), f = m == now ? 1.f : expf(m - now), p = z == now ? 1.f : expf(z - now);
                l = fmaf(l, f, p);
#pragma unroll
                for (int d = 0; d < D / 32; ++d) o[d] = fmaf(p, x[d], o[d] * f);
                m = now;
            }
            const long long to = (s.row + i) * P.o_token + head * P.o_head + lane * (D / 32);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) store_elem<DT>(P.out, to + d, l == 0.f ? 0.f : o[d] / l);
            if (P.lse && lane == 0) P.lse[(s.row + i) * P.n_heads + head] = l == 0.f ? -INFINITY : m + logf(l);
        }
    }
}

// A warp per (position, key head).
template <int DT, int D>
__global__ void __launch_bounds__(256)
weigh_kernel(const __grid_constant__ ChunkParams P)
{
    const int lane = threadIdx.x & 31, head = blockIdx.x, ps = 1 << P.c.page_shift;
    for (int b = blockIdx.y; b < P.batch; b += gridDim.y) {
        const ChunkSeq s = chunk_seq(P, b);
        const int32_t *table = P.table + b * P.ld_table;
        if (s.count == 0) continue;
        const int first = P.last > 0 ? max(s.count - P.last, 0) : 0;
        for (int pos = blockIdx.z * 8 + (threadIdx.x >> 5); pos < s.len; pos += gridDim.z * 8) {
            float k[D / 32];
            if (!chunk_row<D>(P.c, table, pos, head, 0, lane, k)) continue;
            float sum = 0.f;
            for (int i = max(first, pos - s.start); i < s.count; ++i)
                for (int h = head * P.group; h < (head + 1) * P.group; ++h) {
                    const long long at = (s.row + i) * P.q_token + h * P.q_head + lane * (D / 32);
                    float z = 0.f;
#pragma unroll
                    for (int d = 0; d < D / 32; ++d) z = fmaf(load_elem<DT>(P.q, at + d), k[d], z);
                    z = warp_sum(z) * P.scale;
                    const float lse = P.lse[(s.row + i) * P.n_heads + h];
                    if (lse != -INFINITY) sum += expf(z - lse);
                }
            if (lane == 0) {
                float *w = P.weights + (static_cast<long long>(table[pos >> P.c.page_shift]) * P.c.n_heads + head) * ps + (pos & (ps - 1));
                *w = pos < s.start && P.decay != 0.f ? fmaf(P.decay, *w, sum) : sum;
            }
        }
    }
}

}  // namespace mcsd
