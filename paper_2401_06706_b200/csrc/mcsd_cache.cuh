// The paged key/value cache in 4 bits: append_kernel quantises rows and stores them at their slots,
// read_kernel reads them back, move_kernel moves the rows of the accepted path.  The layout of a page
// is the one mcsd.h documents.
#pragma once

#include "mcsd_common.cuh"

namespace mcsd {

// Bytes of the block of one head in one page and where its parts begin.
__host__ __device__ __forceinline__ constexpr int kv_block_bytes(int dim, int page_size) { return page_size * (dim + 8); }

struct CacheParams {
    unsigned char *pages;
    long long page_stride;                          // bytes
    int32_t n_pages, n_heads, page_shift;
};

struct RowsParams {
    CacheParams c;
    void *keys, *values;                            // (read only in append_kernel); a null one is skipped
    long long key_token, key_head, value_token, value_head;  // strides in elements
    const long long *slots;
    long long n_tokens;
};

// Where row `which` (0 key, 1 value) of (token slot, head) lies; false if the slot is not in the cache.
template <int D>
__device__ __forceinline__ bool kv_row(const CacheParams &c, long long slot, int head, int which, unsigned char *&codes,
                                       __half2 *&param)
{
    const long long page = slot >> c.page_shift;
    if (slot < 0 || page >= c.n_pages) return false;
    const int ps = 1 << c.page_shift, row = static_cast<int>(slot) & (ps - 1);
    unsigned char *block = c.pages + page * c.page_stride + static_cast<long long>(head) * kv_block_bytes(D, ps);
    codes = block + (which * ps + row) * (D / 2);
    param = reinterpret_cast<__half2 *>(block + ps * D) + which * ps + row;
    return true;
}

// A group of D / 8 threads keeps one row of every token (a key or a value row of one head) and steps over
// the tokens: with 2 n_heads groups per token, group i of the grid has row i % (2 n_heads) of tokens
// i / (2 n_heads), that + `step`, ...; groups beyond the last full token of the grid have nothing to do.
struct RowWalk { long long token, step; int which, head; };
template <int TPR>
__device__ __forceinline__ RowWalk row_walk(const RowsParams &P)
{
    const uint32_t rows = 2u * static_cast<uint32_t>(P.c.n_heads);
    const uint32_t groups = gridDim.x * (256u / TPR), mine = (blockIdx.x * 256u + threadIdx.x) / TPR;
    RowWalk w;
    w.step = groups / rows;
    w.token = mine / rows;
    const uint32_t row = mine - static_cast<uint32_t>(w.token) * rows;
    w.which = row >= static_cast<uint32_t>(P.c.n_heads);
    w.head = static_cast<int>(row) - (w.which ? P.c.n_heads : 0);
    if (w.token >= w.step) w.token = P.n_tokens;
    return w;
}

// D / 8 threads per row, 8 numbers each: the row's extremes by shuffles, then every thread rounds its own
// 8 and stores one word of codes.  Rows of a token's heads follow each other in the thread order, so that
// loads are contiguous (a page's rows of one head are 32 to 64 contiguous bytes each).  Bound by HBM: 2 D
// numbers read and D + 8 bytes written per key/value row pair; a thread takes kRowsAhead tokens at a time, so
// that their slots, and then their numbers, are in flight together.  Measured on 40001 tokens x 8 heads x 128 halves: 87 us
// alone, 91 in a pass that reads back as well (0.35 of the measured copy bandwidth; the loads of a thread wait for one another, and some 150
// instructions for the two rows of a warp are the other half of it), the way back 51 us (0.61; every token's codes wait for its slot). Other numbers of tokens at a time: 4 take 94 us, 2 take 98, and
// for the way back 2 take 55 us, 4 take 67; with a grid of eight CTAs per SM (not all resident) 106 and 68 us.
// Scale and mid are formed in double (by one of a row's threads), rounded to float32 and then to half, as the definition says; codes are
// those of exact arithmetic on them: where x / scale - mid / scale in float32 lies within 2^-18 + |mid / scale| 2^-23
// of a border between two codes (a reciprocal good to 2^-23 and the last rounding put a number up to 8.5 off by 2^-18.9 at most,
// the rounding of mid / scale by |mid / scale| 2^-24) the thread's codes are decided in double; so no code depends on
// how the compiler orders things.  Rounding to an integer is an addition of 1.5 2^23 (the conversion
// instructions have a quarter of the rate).
constexpr int kRowsAhead = 3;
constexpr int kAppendCtas = 3, kReadCtas = 6;         // per SM: those that are resident, so that all end at about the same time

// Extremes of a thread's 8 numbers, NaN if one is NaN.
__device__ __forceinline__ float min_nan(float a, float b) { float d; asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
__device__ __forceinline__ float max_nan(float a, float b) { float d; asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
template <int DT> struct Pair;                      // two 16-bit numbers in a word
template <> struct Pair<MCSD_DTYPE_F16> {
    typedef __half2 T;
    static __device__ __forceinline__ T lo(T a, T b) { return __hmin2_nan(a, b); }
    static __device__ __forceinline__ T hi(T a, T b) { return __hmax2_nan(a, b); }
    static __device__ __forceinline__ float2 wide(T a) { return __half22float2(a); }
    static __device__ __forceinline__ T low_and_minus_high(T l, T h) { return __halves2half2(__hmin_nan(__low2half(l), __high2half(l)), __hneg(__hmax_nan(__low2half(h), __high2half(h)))); }
};
template <> struct Pair<MCSD_DTYPE_BF16> {
    typedef __nv_bfloat162 T;
    static __device__ __forceinline__ T lo(T a, T b) { return __hmin2_nan(a, b); }
    static __device__ __forceinline__ T hi(T a, T b) { return __hmax2_nan(a, b); }
    static __device__ __forceinline__ float2 wide(T a) { return __bfloat1622float2(a); }
    static __device__ __forceinline__ T low_and_minus_high(T l, T h) { return __halves2bfloat162(__hmin_nan(__low2bfloat16(l), __high2bfloat16(l)), __hneg(__hmax_nan(__low2bfloat16(h), __high2bfloat16(h)))); }
};

__device__ __forceinline__ float rcp_approx(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// (scale, mid) of a row from its extremes; (0, NaN) if one of them is not finite.
__device__ __forceinline__ uint32_t row_param(float lo, float hi)
{
    if (!(fabsf(lo) <= 3.4028235e38f && fabsf(hi) <= 3.4028235e38f)) return 0x7fff0000u;
    // range / 15, correctly rounded: the quotient by the rounded reciprocal, corrected by its exact remainder (Markstein)
    constexpr double kFifteenth = 1.0 / 15.0;
    const double range = static_cast<double>(hi) - static_cast<double>(lo);
    const double near = range * kFifteenth;
    const double step = fma(fma(-15.0, near, range), kFifteenth, near);
    const __half scale = __float2half_rn(static_cast<float>(fmin(step, 65504.0)));
    const double mid = fma(8.0, static_cast<double>(__half2float(scale)), static_cast<double>(lo));
    const __half2 p = __halves2half2(scale, __float2half_rn(static_cast<float>(fmax(-65504.0, fmin(mid, 65504.0)))));
    return *reinterpret_cast<const uint32_t *>(&p);
}

template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(256, kAppendCtas)
append_kernel(const RowsParams P)
{
    constexpr int TPR = D / 8;                      // threads of a row
    constexpr int kLoads = Elem<DT>::kBytes / 2;
    const int lane = threadIdx.x % TPR;
    const uint32_t group = ((1u << TPR) - 1u) << (threadIdx.x & 31 & ~(TPR - 1));
    const RowWalk walk = row_walk<TPR>(P);
    const char *src = static_cast<const char *>(walk.which ? P.values : P.keys) +
                      (walk.head * (walk.which ? P.value_head : P.key_head) + lane * 8) * Elem<DT>::kBytes;
    const long long pitch = (walk.which ? P.value_token : P.key_token) * Elem<DT>::kBytes;
    for (long long token = walk.token; token < P.n_tokens; token += kRowsAhead * walk.step) {
        unsigned char *codes[kRowsAhead];
        __half2 *param[kRowsAhead];
        uint4 raw[kRowsAhead][kLoads];              // the numbers, in their type
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const long long tok = token + u * walk.step;
            codes[u] = nullptr;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) raw[u][i] = make_uint4(0u, 0u, 0u, 0u);
            if (tok >= P.n_tokens) continue;
            if (!kv_row<D>(P.c, __ldg(P.slots + tok), walk.head, walk.which, codes[u], param[u])) codes[u] = nullptr;
            if constexpr (VEC) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) raw[u][i] = ld_stream_v4(src + tok * pitch + 16 * i);
            } else {
                float x8[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x8[i] = load_elem<DT>(src + tok * pitch, i);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) raw[u][i] = pack_elems<DT>(x8 + i * (8 / kLoads));   // (exact: they come from that type)
            }
        }
        // extremes of the rows; then thread u of a row's forms the two numbers of row u
        float my_lo = 0.f, my_hi = 0.f;
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            float lo, hi;
            if constexpr (DT == MCSD_DTYPE_F32) {
                float x[8];
#pragma unroll
                for (int i = 0; i < kLoads; ++i) Elem<DT>::unpack(raw[u][i], x + i * (8 / kLoads));
                lo = hi = x[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) { lo = min_nan(lo, x[i]); hi = max_nan(hi, x[i]); }
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1) {
                    lo = min_nan(lo, __shfl_xor_sync(group, lo, o));
                    hi = max_nan(hi, __shfl_xor_sync(group, hi, o));
                }
            } else {
                typedef typename Pair<DT>::T T;
                const T *w = reinterpret_cast<const T *>(&raw[u][0]);
                T both = Pair<DT>::low_and_minus_high(Pair<DT>::lo(Pair<DT>::lo(w[0], w[1]), Pair<DT>::lo(w[2], w[3])),
                                                      Pair<DT>::hi(Pair<DT>::hi(w[0], w[1]), Pair<DT>::hi(w[2], w[3])));
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1) {
                    const uint32_t other = __shfl_xor_sync(group, *reinterpret_cast<const uint32_t *>(&both), o);
                    both = Pair<DT>::lo(both, *reinterpret_cast<const T *>(&other));
                }
                const float2 f = Pair<DT>::wide(both);
                lo = f.x;
                hi = -f.y;
            }
            if (lane == u) { my_lo = lo; my_hi = hi; }
        }
        // (the sign of the scale carries whether a number of the row may round beyond codes 0 to 15)
        uint32_t mine = row_param(my_lo, my_hi);
        {
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&mine));
            const float inv = rcp_approx(p.x);
            if (!((my_hi - p.y) * inv < 7.4f && (my_lo - p.y) * inv > -8.4f)) mine |= 0x8000u;
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const uint32_t flagged = __shfl_sync(group, mine, u, TPR), both = flagged & ~0x8000u;
            if (!codes[u]) continue;                // (the same for all threads of the row)
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&both));
            const float s = p.x, m = p.y;
            const float inv = rcp_approx(s), off = m * inv;         // (unused where s is 0)
            float x[8];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) Elem<DT>::unpack(raw[u][i], x + i * (8 / kLoads));
            float2 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = fma2(make_float2(x[2 * i], x[2 * i + 1]), make_float2(inv, inv), make_float2(-off, -off));
            if (flagged & 0x8000u) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    q[i].x = fminf(fmaxf(q[i].x, -8.f), 7.f);
                    q[i].y = fminf(fmaxf(q[i].y, -8.f), 7.f);
                }
            }
            constexpr float kRound = 12582912.f + 8.f;              // 1.5 2^23, and code 8 at 0: a sum's bits are 0x4b400000 + code
            uint32_t word = 0u;
            float far = 0.f;
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                const float2 t = add2(q[i], make_float2(kRound, kRound));
                const float2 d = add2(q[i], make_float2(kRound - t.x, kRound - t.y));  // off the code (the difference is exact)
                far = max3(far, fabsf(d.x), fabsf(d.y));
                word = word * 16u + __float_as_uint(t.y);
                word = word * 16u + __float_as_uint(t.x);
            }
            word -= 0x4b400000u * 0x11111111u;
            if (far > fmaf(fabsf(off), -1.1920929e-7f, 0.5f - 3.814697265625e-6f)) {
                word = 0u;
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const double q = (static_cast<double>(x[0]) - static_cast<double>(m)) / static_cast<double>(s);
                    const double n = fmin(fmax(rint(q), -8.0), 7.0);
                    word = word >> 4 | static_cast<uint32_t>(static_cast<int>(n) + 8) << 28;
#pragma unroll
                    for (int j = 0; j < 7; ++j) x[j] = x[j + 1];
                }
            }
            reinterpret_cast<uint32_t *>(codes[u])[lane] = s > 0.f ? word : 0x88888888u;
            if (lane == 0) *reinterpret_cast<uint32_t *>(param[u]) = both;
        }
    }
}

// The way back, one thread per 8 numbers.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(256, kReadCtas)
read_kernel(const RowsParams P)
{
    constexpr int TPR = D / 8;
    const int lane = threadIdx.x % TPR;
    const RowWalk walk = row_walk<TPR>(P);
    char *out = static_cast<char *>(walk.which ? P.values : P.keys);
    if (!out) return;
    out += (walk.head * (walk.which ? P.value_head : P.key_head) + lane * 8) * Elem<DT>::kBytes;
    const long long pitch = (walk.which ? P.value_token : P.key_token) * Elem<DT>::kBytes;
    for (long long token = walk.token; token < P.n_tokens; token += kRowsAhead * walk.step) {
        char *dst[kRowsAhead];
        __half2 p[kRowsAhead];
        uint32_t word[kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const long long tok = token + u * walk.step;
            dst[u] = nullptr;
            if (tok >= P.n_tokens) continue;
            unsigned char *codes;
            __half2 *param;
            if (!kv_row<D>(P.c, __ldg(P.slots + tok), walk.head, walk.which, codes, param)) continue;
            dst[u] = out + tok * pitch;
            p[u] = *param;
            word[u] = reinterpret_cast<const uint32_t *>(codes)[lane];
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            if (!dst[u]) continue;
            const float2 f = __half22float2(p[u]);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {        // (a code in the mantissa of 2^23: no conversion)
                const float2 c = add2(make_float2(__uint_as_float((word[u] >> (4 * i)) & 15u | 0x4b000000u),
                                                  __uint_as_float((word[u] >> (4 * i + 4)) & 15u | 0x4b000000u)), make_float2(-8388616.f, -8388616.f));
                const float2 y = fma2(make_float2(f.x, f.x), c, make_float2(f.y, f.y));
                x[i] = y.x;
                x[i + 1] = y.y;
            }
            if constexpr (VEC) {
                constexpr int kStores = Elem<DT>::kBytes / 2;
                uint4 *q = reinterpret_cast<uint4 *>(dst[u]);
#pragma unroll
                for (int i = 0; i < kStores; ++i) q[i] = pack_elems<DT>(x + i * (8 / kStores));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) store_elem<DT>(dst[u], i, x[i]);
            }
        }
    }
}

struct MoveParams {
    CacheParams c;
    long long n_layers, layer_stride;
    const int32_t *table, *prefix_len, *path_nodes, *accept_len;
    long long ld_table;
    int32_t max_pages, batch, gamma;
    int32_t layers_per_item;
};

// Sixteen threads per (run of layers, sequence, head): D / 32 of them own 16 bytes of the key codes each, as many
// 16 bytes of the value codes, one the key parameters, one the value parameters.  As in gather_kernel,
// nodes ascend along a path and lie at or behind their destination, so a thread that handles its columns
// in ascending order never reads what it has overwritten; up to kBatch moves in each of kLayers layers are read before
// one is written.
// Where a row lies is the same in every layer, so a thread finds out once (three loads, each from the one before) and
// uses it for its run of layers.  256 sequences, 32 layers, 8 heads: 23 us in a cold capture, 28 us a call; back to back on the same
// rows it was 21 us, with one layer at a time 24 us, with runs of one layer instead of six 35 us. Some 90000 row pairs are four pieces
// of 4 to 64 bytes each there, read and written at unrelated places (about 7 us in whole 32-byte sectors): what a thread has in flight
// bounds it, and of sixteen threads six (D = 64) or ten work.
template <int D>
__global__ void __launch_bounds__(256)
move_kernel(const MoveParams P)
{
    constexpr int kBatch = 4, kLayers = 2, NC = D / 32;
    const int ps = 1 << P.c.page_shift, lane = threadIdx.x & 15;
    const long long n_items = (P.n_layers + P.layers_per_item - 1) / P.layers_per_item * P.batch * P.c.n_heads;
    const bool wide = lane < 2 * NC;                // a column of codes; then two threads with parameters
    if (lane >= 2 * NC + 2) return;
    // offset of this thread's column in a block, and the bytes from one row of it to the next
    const int column = wide ? (lane / NC) * ps * (D / 2) + (lane % NC) * 16 : ps * D + (lane - 2 * NC) * ps * 4;
    const int pitch = wide ? D / 2 : 4;
    for (long long item = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) >> 4; item < n_items;
         item += static_cast<long long>(gridDim.x) * 16) {
        const int head = static_cast<int>(item % P.c.n_heads);
        const long long rest = item / P.c.n_heads;
        const int b = static_cast<int>(rest % P.batch);
        const long long layer0 = rest / P.batch * P.layers_per_item, layer1 = min(layer0 + P.layers_per_item, static_cast<long long>(P.n_layers));
        const int prefix = P.prefix_len[b];
        const int len = min(max(P.accept_len[b], 0), P.gamma);
        if (prefix < 0) continue;
        unsigned char *base = P.c.pages + static_cast<long long>(head) * kv_block_bytes(D, ps) + column;
        const int32_t *nodes = P.path_nodes + static_cast<long long>(b) * (P.gamma + 1);
        const int32_t *table = P.table + b * P.ld_table;
        // offset of a position's row in a layer, -1 where the cache has none
        auto place = [&](long long pos) -> long long {
            const long long j = pos >> P.c.page_shift;
            if (j >= P.max_pages) return -1;
            const int page = __ldg(table + j);
            if (page < 0 || page >= P.c.n_pages) return -1;
            return page * P.c.page_stride + static_cast<int>(pos & (ps - 1)) * pitch;
        };
        for (int i0 = 0; i0 < len; i0 += kBatch) {
            long long from[kBatch], to[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = i0 + u, nd = i < len ? __ldg(nodes + i) : 0;
                // (nd == i + 1 stays where it is, one below cannot come from a walk)
                from[u] = nd > i + 1 ? place(static_cast<long long>(prefix) + nd) : -1;
                to[u] = nd > i + 1 ? place(static_cast<long long>(prefix) + 1 + i) : -1;
            }
            for (long long layer = layer0; layer < layer1; layer += kLayers) {
                uint4 v[kLayers][kBatch];
#pragma unroll
                for (int y = 0; y < kLayers; ++y) {
                    const unsigned char *here = base + (layer + y) * P.layer_stride;
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
                        if (from[u] >= 0 && to[u] >= 0 && layer + y < layer1) {
                            if (wide) v[y][u] = *reinterpret_cast<const uint4 *>(here + from[u]);
                            else v[y][u].x = *reinterpret_cast<const uint32_t *>(here + from[u]);
                        }
                }
#pragma unroll
                for (int y = 0; y < kLayers; ++y) {
                    unsigned char *here = base + (layer + y) * P.layer_stride;
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
                        if (from[u] >= 0 && to[u] >= 0 && layer + y < layer1) {
                            if (wide) *reinterpret_cast<uint4 *>(here + to[u]) = v[y][u];
                            else *reinterpret_cast<uint32_t *>(here + to[u]) = v[y][u].x;
                        }
                }
            }
        }
    }
}

}  // namespace mcsd
