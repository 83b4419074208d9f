// Log probabilities of given tokens, entropy and the largest tokens of rows of logits.
#pragma once

#include "mcsd_common.cuh"

namespace mcsd {

struct LogprobParams {
    const void *logits;
    long long ld, n_logits, n_out;
    const int32_t *row_index, *path_nodes, *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *top_ids;
    int32_t V, n_given, n_top, path_len, nodes_per_tree;
    float inv_t, scale;                             // 1 / T, log2(e) / T
};

constexpr int kLogprobGroups = 64;                  // groups of threads whose maxima give the bar for candidates: at least MCSD_MAX_TOP
constexpr int kLogprobKeys = 1024;                  // candidates that are kept
constexpr float kLogitFloor = -3.402823466e+38f;

// Row of the logits that output row i reads, -1 if none.
__device__ __forceinline__ long long logprob_row(const LogprobParams &P, long long i)
{
    long long r = i;
    if (P.path_nodes) {
        const long long b = i / P.path_len, j = i - b * P.path_len;
        const int node = j == 0 ? 0 : __ldg(P.path_nodes + i - 1);
        if (node < 0 || node >= P.nodes_per_tree) return -1;
        r = b * P.nodes_per_tree + node;
    } else if (P.row_index) {
        r = __ldg(P.row_index + i);
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
__device__ __forceinline__ int key_token(unsigned long long key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

// A row's sums relative to a reference m: z = sum 2^((l - m) scale), e = the same weighted by (l - m) scale.
struct LogprobSums { float m, z, e; };
__device__ __forceinline__ LogprobSums join_sums(const LogprobSums &a, const LogprobSums &b, float scale)
{
    LogprobSums r;
    r.m = fmaxf(a.m, b.m);
    // (an empty side is kLogitFloor away at most: its product with 0 stays one)
    const float da = fmaxf((a.m - r.m) * scale, -1e30f), db = fmaxf((b.m - r.m) * scale, -1e30f);
    const float fa = ex2f(da), fb = ex2f(db);
    r.z = fmaf(fa, a.z, fb * b.z);
    r.e = fmaf(fa, fmaf(da, a.z, a.e), fb * fmaf(db, b.z, b.e));
    return r;
}

// One CTA per row, one pass over it: each thread keeps sums relative to its own running maximum (a batch of 64 bytes has
// one correction), which a tree of shuffles joins. For the largest tokens that maximum is all that the pass costs: the n-th
// largest of the 64 group maxima is reached by n elements at least, so that only threads whose own maximum reaches it look at their
// elements again (from L2) and hand those that do to a list, of which the n first are taken by counting. A row whose list
// overflows is searched n times instead, element by element: one with many equal logits, and one in which fewer than n groups have a finite
// logit, so that the bar is -inf or the value of a mask (few allowed tokens; short 16-bit rows on 1024 threads, whose groups are neighbours). That is slow: 98 instead of 14 us for 8 rows of 32000 bf16
// logits with 20 allowed and 20 asked for, 480 instead of 39 for 1021 of them, 46 for 8 rows of 2000 (12 in fp32).
// Sums of a thread (V / THREADS terms) and their joining are float32: an error of 2^-22 of the result or so; a distance from the maximum
// is formed before it is scaled, so that the lowest finite logits (a mask) do not overflow against one another.
// Bound by the reading of the logits and by the tail of a row (joining, candidates), in which a CTA reads nothing; eight CTAs an SM overlap that: 1021 rows of
// 50272 fp32 logits, 8 tokens: 54 us where a part comes from L2, 77 from HBM (2.7 of 6.55 TB/s); 2047 rows of 32000 bf16, 20 tokens: 53 and 68. A CTA per row instead
// of a loop over rows 75 -> 54; a maximum and the candidates in a pass of their own 97 (fp32).
template <int DT, int THREADS, bool VEC>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 1 : 8)
logprob_kernel(const __grid_constant__ LogprobParams P)
{
    typedef Elem<DT> E;
    constexpr int KV = E::kVec, BATCH = 4, WARPS = THREADS / 32, PER_GROUP = THREADS / kLogprobGroups;
    __shared__ LogprobSums s_sums[WARPS];
    __shared__ __align__(16) float s_top[kLogprobGroups];
    __shared__ float s_bar;
    __shared__ int s_count;
    __shared__ unsigned long long s_keys[kLogprobKeys];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float scale = P.scale, none = __int_as_float(0x7fc00000);

    const long long i = blockIdx.x, r = logprob_row(P, i);
    if (r < 0) return;                          // (the same for the whole CTA)
    const char *row = static_cast<const char *>(P.logits) + r * P.ld * E::kBytes;
    const int vectors = VEC ? P.V / KV : 0;     // (what is left of a row goes element by element)

    LogprobSums mine = {kLogitFloor, 0.f, 0.f};
    float most = -INFINITY;                     // of the thread's logits
    float2 z2 = make_float2(0.f, 0.f), e2 = make_float2(0.f, 0.f);
    auto move_to = [&](float m) {               // a new reference
        const float d = fmaxf((mine.m - m) * scale, -1e30f), f = ex2f(d);
        e2 = __fmul2_rn(fma2(make_float2(d, d), z2, e2), make_float2(f, f));
        z2 = __fmul2_rn(z2, make_float2(f, f));
        mine.m = m;
    };
    auto add_pair = [&](float x, float y) {
        float2 d = __fmul2_rn(add2(make_float2(x, y), make_float2(-mine.m, -mine.m)), make_float2(scale, scale));
        asm("max.NaN.f32 %0, %0, 0fc3480000;" : "+f"(d.x));        // -200: its power is 0, its product with that too
        asm("max.NaN.f32 %0, %0, 0fc3480000;" : "+f"(d.y));
        const float2 p = make_float2(ex2f(d.x), ex2f(d.y));
        z2 = add2(z2, p);
        e2 = fma2(p, d, e2);
    };
    for (int v0 = tid; v0 < vectors; v0 += THREADS * BATCH) {
        uint4 raw[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
            raw[u] = ld_stream_v4_if(row + static_cast<long long>(v0 + u * THREADS) * 16, v0 + u * THREADS < vectors, E::kNegInfWord);
        typename E::MaxAcc acc = E::max_init();
#pragma unroll
        for (int u = 0; u < BATCH; ++u) E::max_step(acc, raw[u]);
        const float top = E::max_final(acc);
        most = fmaxf(most, top);
        if (top > mine.m) move_to(top);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            float x[KV];
            E::unpack(raw[u], x);
#pragma unroll
            for (int j = 0; j < KV; j += 2) add_pair(x[j], x[j + 1]);
        }
    }
    for (int x = vectors * KV + tid; x < P.V; x += THREADS) {
        const float l = E::load(row, x);
        most = fmaxf(most, l);
        if (l > mine.m) move_to(l);
        add_pair(l, -INFINITY);
    }
    mine.z = z2.x + z2.y;
    mine.e = e2.x + e2.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        LogprobSums other;
        other.m = __shfl_xor_sync(0xffffffffu, mine.m, o);
        other.z = __shfl_xor_sync(0xffffffffu, mine.z, o);
        other.e = __shfl_xor_sync(0xffffffffu, mine.e, o);
        mine = join_sums(mine, other, scale);
    }
    if (lane == 0) s_sums[warp] = mine;
    if (P.n_top > 0) {
        float group = most;
#pragma unroll
        for (int o = 1; o < PER_GROUP; o <<= 1) group = fmaxf(group, __shfl_xor_sync(0xffffffffu, group, o));
        if (tid % PER_GROUP == 0) s_top[tid / PER_GROUP] = group;
        if (tid == 0) s_count = 0;
    }
    __syncthreads();
    mine = s_sums[0];
    for (int w = 1; w < WARPS; ++w) mine = join_sums(mine, s_sums[w], scale);
    // (no mass, or a NaN or infinite logit in it: no distribution)
    const bool sound = mine.z > 0.f && mine.z < INFINITY;
    const float log_z = sound ? logf(mine.z) : none;
    auto logprob = [&](float l) { return fmaf(l - mine.m, P.inv_t, -log_z); };
    if (tid == 0 && P.entropy) P.entropy[i] = sound ? fmaxf(fmaf(-0.6931471805599453f, mine.e / mine.z, log_z), 0.f) : none;
    if (P.logprobs)
        for (int g = tid; g < P.n_given; g += THREADS) {
            const int x = __ldg(P.tokens + i * P.n_given + g);
            P.logprobs[i * P.n_given + g] = x < 0 || x >= P.V || !sound ? none : logprob(E::load(row, x));
        }
    if (P.n_top > 0 && !sound) {
        for (int k = tid; k < P.n_top; k += THREADS) {
            if (P.top_ids) P.top_ids[i * P.n_top + k] = -1;
            if (P.top_logprobs) P.top_logprobs[i * P.n_top + k] = none;
        }
    } else if (P.n_top > 0) {
        if (tid < kLogprobGroups) {             // the n_top-th largest of the group maxima
            const float own = s_top[tid];
            int rank = 0;
#pragma unroll
            for (int g = 0; g < kLogprobGroups; g += 4) {
                const float4 o = *reinterpret_cast<const float4 *>(s_top + g);
                rank += (o.x > own || (o.x == own && g < tid)) + (o.y > own || (o.y == own && g + 1 < tid)) +
                        (o.z > own || (o.z == own && g + 2 < tid)) + (o.w > own || (o.w == own && g + 3 < tid));
            }
            if (rank == P.n_top - 1) s_bar = own;
        }
        __syncthreads();
        const float bar = s_bar;
        auto offer = [&](float l, int x) {
            if (l >= bar) {
                const int at = atomicAdd(&s_count, 1);
                if (at < kLogprobKeys) s_keys[at] = logit_key(l, x);
            }
        };
        if (most >= bar) {
            for (int v = tid; v < vectors; v += THREADS) {
                float x[KV];
                E::unpack(ld_v4_if(row + static_cast<long long>(v) * 16, true, 0u), x);
#pragma unroll
                for (int j = 0; j < KV; ++j) offer(x[j], v * KV + j);
            }
            for (int x = vectors * KV + tid; x < P.V; x += THREADS) offer(E::load(row, x), x);
        }
        __syncthreads();
        const int n = s_count;
        if (n <= kLogprobKeys) {
            for (int k = tid; k < n; k += THREADS) {
                const unsigned long long key = s_keys[k];
                int rank = 0;
                for (int o = 0; o < n; ++o) rank += s_keys[o] > key;
                if (rank < P.n_top) {
                    const int x = key_token(key);
                    if (P.top_ids) P.top_ids[i * P.n_top + rank] = x;
                    if (P.top_logprobs) P.top_logprobs[i * P.n_top + rank] = logprob(E::load(row, x));
                }
            }
        } else {
            unsigned long long last = ~0ull;
            for (int k = 0; k < P.n_top; ++k) {
                unsigned long long best = 0ull;
                for (int x = tid; x < P.V; x += THREADS) {
                    const unsigned long long key = logit_key(E::load(row, x), x);
                    if (key < last && key > best) best = key;
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
                    best = best > other ? best : other;
                }
                __syncthreads();
                if (lane == 0) s_keys[warp] = best;
                __syncthreads();
                for (int w = 0; w < WARPS; ++w) best = best > s_keys[w] ? best : s_keys[w];
                if (tid == 0) {
                    const int x = key_token(best);
                    if (P.top_ids) P.top_ids[i * P.n_top + k] = x;
                    if (P.top_logprobs) P.top_logprobs[i * P.n_top + k] = logprob(E::load(row, x));
                }
                last = best;
            }
        }
    }
}

}  // namespace mcsd
