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
    uint32_t n_rows;                                // tokens * heads * 2
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

// Row r of a call: its token, whether it is a value row, and its head; rows of a token's heads follow each other.
struct RowIndex { uint32_t token; int which, head; };
__device__ __forceinline__ RowIndex row_index(const RowsParams &P, uint32_t r)
{
    RowIndex x;
    const uint32_t rest = r / static_cast<uint32_t>(P.c.n_heads);
    x.head = static_cast<int>(r - rest * static_cast<uint32_t>(P.c.n_heads));
    x.which = static_cast<int>(rest & 1u);
    x.token = rest >> 1;
    return x;
}

// D / 8 threads per row, 8 numbers each: the row's extremes by shuffles, then every thread rounds its own
// 8 and stores one word of codes.  Rows of a token's heads follow each other in the thread order, so that
// loads are contiguous (a page's rows of one head are 32 to 64 contiguous bytes each).  Bound by HBM: 2 D
// numbers read and D + 8 bytes written per key/value row pair; a thread takes kRowsAhead rows at a time, so
// that their slots, and then their numbers, are in flight together.
// Scale, mid and codes are those of the definition in exact arithmetic: the two per-row numbers are formed
// in double (once a row), and a code whose float32 quotient lies within 2^-10 of a border between two codes
// (float32 is off by a few 2^-20 at most) is decided in double; so no code depends on how the compiler orders things.
constexpr int kRowsAhead = 4;

template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(256)
append_kernel(const RowsParams P)
{
    constexpr int TPR = D / 8;                      // threads of a row
    constexpr int kLoads = Elem<DT>::kBytes / 2;
    const uint32_t stride = gridDim.x * (256 / TPR);
    const int lane = threadIdx.x % TPR;
    const uint32_t group = ((1u << TPR) - 1u) << (threadIdx.x & 31 & ~(TPR - 1));
    for (uint32_t r0 = (blockIdx.x * 256 + threadIdx.x) / TPR; r0 < P.n_rows;) {
        unsigned char *codes[kRowsAhead];
        __half2 *param[kRowsAhead];
        uint4 raw[kRowsAhead][VEC ? kLoads : 1];
        long long at[kRowsAhead];
        const void *src[kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const uint32_t r = r0 + u * stride;     // (far below 2^32: the host bounds the rows)
            codes[u] = nullptr;
            if (r >= P.n_rows) continue;
            const RowIndex x = row_index(P, r);
            if (!kv_row<D>(P.c, __ldg(P.slots + x.token), x.head, x.which, codes[u], param[u])) codes[u] = nullptr;
            src[u] = x.which ? P.values : P.keys;
            at[u] = (x.which ? x.token * P.value_token + x.head * P.value_head : x.token * P.key_token + x.head * P.key_head) + lane * 8;
            if constexpr (VEC) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) raw[u][i] = ld_stream_v4(static_cast<const char *>(src[u]) + at[u] * Elem<DT>::kBytes + 16 * i);
            }
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            if (!codes[u]) continue;                // (the same for all threads of the row)
            float x[8];
            if constexpr (VEC) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) Elem<DT>::unpack(raw[u][i], x + i * (8 / kLoads));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = load_elem<DT>(src[u], at[u] + i);
            }
            float lo = x[0], hi = x[0], odd = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo = fminf(lo, x[i]);
                hi = fmaxf(hi, x[i]);
                odd += x[i] * 0.f;                  // NaN if any number is infinite or NaN
            }
#pragma unroll
            for (int o = TPR / 2; o > 0; o >>= 1) {
                lo = fminf(lo, __shfl_xor_sync(group, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(group, hi, o));
            }
            const bool bad = (__ballot_sync(group, !(odd == 0.f)) & group) != 0u;
            // range / 15, correctly rounded: the quotient by the rounded reciprocal, corrected by its exact remainder (Markstein)
            constexpr double kFifteenth = 1.0 / 15.0;
            const double range = static_cast<double>(hi) - static_cast<double>(lo);
            const double near = range * kFifteenth;
            const double step = fma(fma(-15.0, near, range), kFifteenth, near);
            const __half scale = __float2half_rn(static_cast<float>(fmin(step, 65504.0)));
            const float s = __half2float(scale);
            const __half mid = __float2half_rn(static_cast<float>(fmax(-65504.0, fmin(fma(8.0, static_cast<double>(s), static_cast<double>(lo)), 65504.0))));
            const float m = __half2float(mid);
            const float inv = s > 0.f ? 1.f / s : 0.f;
            uint32_t word = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float q = (x[i] - m) * inv;
                float n = rintf(q);
                // near a border (or where the difference itself may have rounded) the quotient is formed in double
                if (fabsf(fabsf(q - n) - 0.5f) < 0.0009765625f)
                    n = static_cast<float>(rint((static_cast<double>(x[i]) - static_cast<double>(m)) / static_cast<double>(s)));
                n = fminf(fmaxf(n, -8.f), 7.f);
                word |= static_cast<uint32_t>(static_cast<int>(n) + 8) << (4 * i);
            }
            reinterpret_cast<uint32_t *>(codes[u])[lane] = !bad && s > 0.f ? word : 0x88888888u;
            if (lane == 0) *param[u] = bad ? __halves2half2(__ushort_as_half(0), __ushort_as_half(0x7fff)) : __halves2half2(scale, mid);
        }
        if (P.n_rows - r0 <= kRowsAhead * stride) break;
        r0 += kRowsAhead * stride;
    }
}

// The way back, one thread per 8 numbers.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(256)
read_kernel(const RowsParams P)
{
    constexpr int TPR = D / 8;
    const uint32_t stride = gridDim.x * (256 / TPR);
    const int lane = threadIdx.x % TPR;
    for (uint32_t r0 = (blockIdx.x * 256 + threadIdx.x) / TPR; r0 < P.n_rows;) {
        void *dst[kRowsAhead];
        long long at[kRowsAhead];
        __half2 p[kRowsAhead];
        uint32_t word[kRowsAhead];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const uint32_t r = r0 + u * stride;
            dst[u] = nullptr;
            if (r >= P.n_rows) continue;
            const RowIndex x = row_index(P, r);
            dst[u] = x.which ? P.values : P.keys;
            unsigned char *codes;
            __half2 *param;
            if (!dst[u] || !kv_row<D>(P.c, __ldg(P.slots + x.token), x.head, x.which, codes, param)) { dst[u] = nullptr; continue; }
            at[u] = (x.which ? x.token * P.value_token + x.head * P.value_head : x.token * P.key_token + x.head * P.key_head) + lane * 8;
            p[u] = *param;
            word[u] = reinterpret_cast<const uint32_t *>(codes)[lane];
        }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            if (!dst[u]) continue;
            const float2 f = __half22float2(p[u]);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf(f.x, static_cast<float>((word[u] >> (4 * i)) & 15u) - 8.f, f.y);
            if constexpr (VEC) {
                constexpr int kStores = Elem<DT>::kBytes / 2;
                uint4 *q = reinterpret_cast<uint4 *>(static_cast<char *>(dst[u]) + at[u] * Elem<DT>::kBytes);
#pragma unroll
                for (int i = 0; i < kStores; ++i) q[i] = pack_elems<DT>(x + i * (8 / kStores));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) store_elem<DT>(dst[u], at[u] + i, x[i]);
            }
        }
        if (P.n_rows - r0 <= kRowsAhead * stride) break;
        r0 += kRowsAhead * stride;
    }
}

struct MoveParams {
    CacheParams c;
    long long n_layers, layer_stride;
    const int32_t *table, *prefix_len, *path_nodes, *accept_len;
    long long ld_table;
    int32_t max_pages, batch, gamma;
};

// Sixteen threads per (layer, sequence, head): D / 32 of them own 16 bytes of the key codes each, as many
// 16 bytes of the value codes, one the key parameters, one the value parameters.  As in gather_kernel,
// nodes ascend along a path and lie at or behind their destination, so a thread that handles its columns
// in ascending order never reads what it has overwritten; up to kBatch moves are read before one is written.
template <int D>
__global__ void __launch_bounds__(256)
move_kernel(const MoveParams P)
{
    constexpr int kBatch = 8, NC = D / 32;
    const int ps = 1 << P.c.page_shift, lane = threadIdx.x & 15;
    const long long n_items = P.n_layers * P.batch * P.c.n_heads;
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
        const long long layer = rest / P.batch;
        const int prefix = P.prefix_len[b];
        const int len = min(max(P.accept_len[b], 0), P.gamma);
        if (prefix < 0) continue;
        unsigned char *base = P.c.pages + layer * P.layer_stride + static_cast<long long>(head) * kv_block_bytes(D, ps) + column;
        const int32_t *nodes = P.path_nodes + static_cast<long long>(b) * (P.gamma + 1);
        const int32_t *table = P.table + b * P.ld_table;
        auto place = [&](long long pos) -> unsigned char * {
            const long long j = pos >> P.c.page_shift;
            if (j >= P.max_pages) return nullptr;
            const int page = table[j];
            if (page < 0 || page >= P.c.n_pages) return nullptr;
            return base + page * P.c.page_stride + static_cast<int>(pos & (ps - 1)) * pitch;
        };
        for (int i0 = 0; i0 < len; i0 += kBatch) {
            uint4 v[kBatch];
            unsigned char *to[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = i0 + u;
                to[u] = nullptr;
                if (i < len) {
                    const int nd = nodes[i];
                    if (nd > i + 1) {               // (nd == i + 1 stays where it is, one below cannot come from a walk)
                        const unsigned char *from = place(static_cast<long long>(prefix) + nd);
                        to[u] = from ? place(static_cast<long long>(prefix) + 1 + i) : nullptr;
                        if (to[u]) {
                            if (wide) v[u] = *reinterpret_cast<const uint4 *>(from);
                            else v[u].x = *reinterpret_cast<const uint32_t *>(from);
                        }
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (to[u]) {
                    if (wide) *reinterpret_cast<uint4 *>(to[u]) = v[u];
                    else *reinterpret_cast<uint32_t *>(to[u]) = v[u].x;
                }
        }
    }
}

}  // namespace mcsd
