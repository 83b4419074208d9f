// Attention of a flattened draft tree over the paged 4-bit cache.
#pragma once

#include "mcsd_cache.cuh"

namespace mcsd {

constexpr int kAttUnit = 128;                       // keys of one unit of work

struct AttendParams {
    CacheParams c;
    const void *q;
    void *out;
    float *lse;                                     // may be null
    float *part;                                    // partial results, two slots per CTA
    const int32_t *table, *prefix_len;
    long long ld_table;
    long long q_seq, q_node, q_head, o_seq, o_node, o_head;  // strides in elements
    int32_t batch, n_nodes, n_heads, max_pages;
    int32_t group;                                  // query heads per key/value head
    int32_t n_rows;                                 // n_nodes * group: rows that share a key/value head
    int32_t n_blocks;                               // blocks of rows per key/value head
    int32_t n_ctas;                                 // CTAs the work is cut for
    int32_t q_vec;                                  // q rows may be read in 16-byte vectors
    float scale;
    int16_t parent[MCSD_MAX_NODES];
};

// ---- the cut of the work
// An item is a block of rows of one (sequence, key/value head); a unit is kAttUnit of its keys.  The
// units of all items, one sequence after the other, are cut into equal runs, one per CTA, so that
// unequal lengths keep every SM busy for the same time.  The lengths are read on the device: a
// captured call follows them.
__device__ __forceinline__ int att_len(const AttendParams &P, int b)
{
    const int prefix = P.prefix_len[b];
    const long long there = static_cast<long long>(P.max_pages) << P.c.page_shift;
    return prefix < 0 ? -1 : static_cast<int>(min(static_cast<long long>(prefix) + P.n_nodes, there));
}
__device__ __forceinline__ int att_units(int len) { return len < 0 ? 0 : max((len + kAttUnit - 1) / kAttUnit, 1); }

// Units before sequence `stop` (all of them for stop == batch) of one item per sequence; every lane gets the sum.
__device__ __forceinline__ long long att_units_before(const AttendParams &P, int stop, int lane)
{
    int sum = 0;                                    // (batch * positions / 128 of a cache that exists: far below 2^31)
    for (int b = lane; b < stop; b += 32) sum += att_units(att_len(P, b));
    return static_cast<long long>(__reduce_add_sync(0xffffffffu, sum));
}

// Position in the cut: the sequence and the unit within its items.
struct AttCursor { int b, len, units; long long at; };

// The sequence that holds unit `u` (in units of all items); u must be below the total.
__device__ __forceinline__ AttCursor att_find(const AttendParams &P, long long u, int items, int lane)
{
    AttCursor c;
    long long before = 0;
    for (int b0 = 0;; b0 += 32) {
        const int b = b0 + lane;
        const int len = b < P.batch ? att_len(P, b) : -1;
        const int n = att_units(len);
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        const unsigned past = __ballot_sync(0xffffffffu, (before + incl) * items > u);
        if (past || b0 + 32 >= P.batch) {
            const int who = past ? __ffs(past) - 1 : 31;
            c.b = b0 + who;
            c.units = __shfl_sync(0xffffffffu, n, who);
            c.len = __shfl_sync(0xffffffffu, len, who);
            c.at = u - (before + __shfl_sync(0xffffffffu, incl - n, who)) * items;
            return c;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
}

// ---- few rows: warp-level matrix instructions on codes that go from shared memory to registers
constexpr int kNarrowWarps = 4, kNarrowStages = 4, kNarrowRows = 16, kNarrowKeys = 32;
template <int D> constexpr int kNarrowStageBytes = kNarrowKeys * (D + 8);
template <int D> constexpr int kNarrowSmem = kNarrowWarps * kNarrowStages * kNarrowStageBytes<D>;
template <int D> constexpr int kPartFloats = kNarrowRows * (D + 2);     // a partial result: rows x D, maxima, sums

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there) {
    const int n = there ? 16 : 0;                   // (0: the 16 bytes are zeros and nothing is read)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Four warps; a warp takes every fourth chunk of 32 keys of the CTA's run with running maxima, sums and
// weighted sums of its own, so that nothing but the end of an item joins them.
//
// The codes never become numbers in memory.  A 4-bit code c in the lowest bits of a half is the subnormal
// number c 2^-24, one in bits 4 to 7 is 16 c 2^-24: one AND turns eight codes of a word into operands of
// the matrix instruction (two at a time), exactly; Q carries the 1/16 of the odd codes, the end of the item that of the
// odd columns.  With mid and scale of a row,
//   <q, k_j> = scale_j sum q c_j + (mid_j - 8 scale_j) sum q
//   sum_j p_j v_j = sum_j (p_j vscale_j) c_j - 8 sum_j (p_j vscale_j) + sum_j p_j vmid_j
// where p vscale is rounded to half once and both of its sums (the second by a matrix instruction against ones)
// use the rounded weight; scores, maxima, sums and the rest are float32.  Q is scaled by a power of two per row so
// that no type's range matters; value scales are taken relative to a power of two E, raised when a larger one comes.
// Weights may exceed 1 by 2^kNarrowSlack before the maximum is moved: the accumulators are rescaled seldom.
//
// Column c of a tile of eight keys is key kappa(c): with this order (and 16-byte chunks of rows 4 to 7 exchanged where a row has
// four) every shared-memory load of codes touches each bank once.
constexpr float kNarrowSlack = 4.f;

template <int DT, int D>
__global__ void __launch_bounds__(kNarrowWarps * 32, 3)
narrow_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int NT = D / 8;                       // n8 tiles of the output
    constexpr int KS = D / 16;                      // k16 steps of the scores
    constexpr int JW = D / 32;                      // words of codes a lane holds of a key row
    constexpr int RB = D / 2;                       // bytes of a code row
    extern __shared__ __align__(128) unsigned char s_ring[];
    __shared__ uint32_t s_seen[kNarrowRows][MCSD_MAX_NODES / 32];
    __shared__ float s_top[kNarrowWarps][kNarrowRows], s_sum[kNarrowWarps][kNarrowRows];
    __shared__ int s_valid[kNarrowWarps][kNarrowStages];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int ps = 1 << P.c.page_shift;
    const int items = P.c.n_heads * P.n_blocks;
    const long long total = att_units_before(P, P.batch, lane) * items;
    const long long per = max((total + P.n_ctas - 1) / P.n_ctas, 1LL);
    long long u = static_cast<long long>(blockIdx.x) * per;
    const long long u_end = min(u + per, total);
    if (u >= u_end) return;
    AttCursor cur = att_find(P, u, items, lane);
    unsigned char *ring = s_ring + warp * kNarrowStages * kNarrowStageBytes<D>;
    auto kappa = [](int c) { return D == 128 ? c ^ ((c >> 1) & 1) : c ^ ((c >> 2) & 1); };
    auto swizzle = [](int row, int chunk) { return D == 128 ? chunk ^ ((row >> 1) & 2) : chunk; };

    while (u < u_end) {
        const int item = static_cast<int>(cur.at / cur.units);
        const int k0 = static_cast<int>(cur.at - static_cast<long long>(item) * cur.units);
        const int k1 = static_cast<int>(min(static_cast<long long>(cur.units), k0 + (u_end - u)));
        const int b = cur.b, len = cur.len, head = item / P.n_blocks, block = item - head * P.n_blocks;
        const int row0 = block * kNarrowRows;
        const int prefix = P.prefix_len[b];
        const bool whole = k0 == 0 && k1 == cur.units;

        __syncthreads();                            // the shared memory of the item before is free
        if (tid < kNarrowRows) {
            for (int i = 0; i * 32 < P.n_nodes; ++i) s_seen[tid][i] = 0u;
            int a = row0 + tid < P.n_rows ? (row0 + tid) / P.group : -1;
            while (a >= 0) {
                s_seen[tid][a >> 5] |= 1u << (a & 31);
                a = P.parent[a];
            }
        }
        // queries: this lane's numbers of rows g and g + 8, scaled to the top of half's range
        uint32_t qa[KS][4];
        float ra[2], rb[2];                         // log2-units per unit of an accumulator; and per unit of (mid - 8 scale)
#pragma unroll
        for (int hrow = 0; hrow < 2; ++hrow) {
            const int r = row0 + g + 8 * hrow;
            float x[D / 4];
#pragma unroll
            for (int i = 0; i < D / 4; ++i) x[i] = 0.f;
            if (r < P.n_rows) {
                const int node = r / P.group, h = head * P.group + (r - node * P.group);
                const long long at = b * P.q_seq + node * P.q_node + h * P.q_head + t * (D / 4);
                if (P.q_vec) {
                    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const char *>(P.q) + at * 2);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) Elem<DT>::unpack(__ldg(src + i), x + 8 * i);
                } else {
#pragma unroll
                    for (int i = 0; i < D / 4; ++i) x[i] = load_elem<DT>(P.q, at + i);
                }
            }
            float top = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 4; ++i) { top = fmaxf(top, fabsf(x[i])); sum += x[i]; }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            }
            // 2^e > top >= 2^(e - 1); the row is scaled by 2^(15 - e)
            int e = top > 0.f ? static_cast<int>(__float_as_uint(top) >> 23) - 126 : 0;
            e = max(min(e, 112), -110);
            const float up = __int_as_float((127 + 15 - e) << 23);
            const float log2e = P.scale * 1.4426950408889634f;
            ra[hrow] = ldexpf(log2e, e - 15 + 24);
            rb[hrow] = log2e * sum;
#pragma unroll
            for (int j = 0; j < JW; ++j)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    qa[2 * j + s][hrow] = half2_bits(x[8 * j + 2 * s] * up, x[8 * j + 2 * s + 4] * up);
                    qa[2 * j + s][2 + hrow] = half2_bits(x[8 * j + 2 * s + 1] * up * 0.0625f, x[8 * j + 2 * s + 5] * up * 0.0625f);
                }
        }
        __syncthreads();

        // this warp's chunks: keys [128 k + 32 warp, + 32) for k = k0 .. k1 - 1, as far as there are keys
        const int left = len - (k0 * kAttUnit + warp * kNarrowKeys);
        const int n_chunks = left <= 0 ? 0 : min(k1 - k0, (left + kAttUnit - 1) / kAttUnit);
        const int32_t *table = P.table + b * P.ld_table;
        const unsigned char *pool = P.c.pages + static_cast<long long>(head) * kv_block_bytes(D, ps);
        // page of this lane's half (16 keys) of chunk i, -1 where there is none
        auto page_of = [&](int i) {
            if (i >= n_chunks) return -1;
            const int pos = (k0 + i) * kAttUnit + warp * kNarrowKeys + (lane & 1) * 16;
            const int j = pos >> P.c.page_shift;
            return pos < len && j < P.max_pages ? table[j] : -1;
        };
        int page_next = page_of(0);
        auto issue = [&](int i) {
            const int page = page_next;
            page_next = page_of(i + 1);             // (its load is in flight while the next chunk is computed)
            if (i < n_chunks) {
                const uint32_t stage = smem_u32(ring + (i % kNarrowStages) * kNarrowStageBytes<D>);
                int ok = 0;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int p = __shfl_sync(0xffffffffu, page, hf);
                    const bool there = p >= 0 && p < P.c.n_pages;
                    ok |= there ? 1 << hf : 0;
                    const int row = ((k0 + i) * kAttUnit + warp * kNarrowKeys + hf * 16) & (ps - 1);
                    const unsigned char *src = pool + (there ? p : 0) * P.c.page_stride;
                    const unsigned char *from = there ? src : P.c.pages;
                    constexpr int CH = RB / 16;     // 16-byte chunks of a row
#pragma unroll
                    for (int n = 0; n < CH / 2; ++n) {
                        const int x = lane + 32 * n, r = x / CH, c = x % CH;
                        const uint32_t dst = stage + (hf * 16 + r) * RB + swizzle(r, c) * 16;
                        cp_async16(dst, there ? src + (row + r) * RB + c * 16 : from, there);
                        cp_async16(dst + kNarrowKeys * RB, there ? src + (ps + row + r) * RB + c * 16 : from, there);
                    }
                    if (lane < 8) {                 // (scale, mid): 64 bytes of the keys, 64 of the values
                        const int which = lane >> 2, c = lane & 3;
                        cp_async16(stage + kNarrowKeys * D + which * kNarrowKeys * 4 + hf * 64 + c * 16,
                                   there ? src + ps * D + which * ps * 4 + row * 4 + c * 16 : from, there);
                    }
                }
                if (lane == 0) s_valid[warp][i % kNarrowStages] = ok;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };

        float o[NT][4], ones[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f}, mids[2] = {0.f, 0.f};
        int expo = -100;                            // value scales are taken in units of 2^expo
#pragma unroll
        for (int i = 0; i < kNarrowStages - 1; ++i) issue(i);
        for (int i = 0; i < n_chunks; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kNarrowStages - 2) : "memory");
            __syncwarp();                           // every lane's copies of chunk i are there, and chunk i - 1 is done with
            const unsigned char *stage = ring + (i % kNarrowStages) * kNarrowStageBytes<D>;
            const int valid = s_valid[warp][i % kNarrowStages];
            issue(i + kNarrowStages - 1);
            const int pos0 = (k0 + i) * kAttUnit + warp * kNarrowKeys;

            float s[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
                const int row = 8 * j + kappa(g);
                uint32_t w[JW];
                if constexpr (D == 128) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(stage + row * RB + swizzle(row, t) * 16);
                    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2 *>(stage + row * RB + t * 8);
                    w[0] = v.x; w[1] = v.y;
                }
#pragma unroll
                for (int n = 0; n < JW; ++n) {
                    const uint32_t y = w[n] >> 8;
                    mma_f16(s[j], qa[2 * n], w[n] & 0x000f000fu, w[n] & 0x00f000f0u);
                    mma_f16(s[j], qa[2 * n + 1], y & 0x000f000fu, y & 0x00f000f0u);
                }
            }
            const __half2 *kp = reinterpret_cast<const __half2 *>(stage + kNarrowKeys * D);
            const __half2 *vp = kp + kNarrowKeys;
            const int ka = kappa(2 * t), kb = kappa(2 * t + 1);
            const bool plain = valid == 3 && pos0 + kNarrowKeys <= prefix;   // every row sees every key
            float2 vs[4], vm[4];                    // (of keys ka, kb)
            float most[2] = {-INFINITY, -INFINITY}, big = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float2 a = __half22float2(kp[8 * j + ka]), c = __half22float2(kp[8 * j + kb]);
                float2 x = __half22float2(vp[8 * j + ka]), y = __half22float2(vp[8 * j + kb]);
                if (!plain) {
                    const int pa = pos0 + 8 * j + ka, pb = pos0 + 8 * j + kb;
                    const bool ta = pa < len && ((valid >> (j >> 1)) & 1), tb = pb < len && ((valid >> (j >> 1)) & 1);
                    if (!ta) { a = make_float2(0.f, 0.f); x = a; }
                    if (!tb) { c = make_float2(0.f, 0.f); y = c; }
                }
                a.y = fmaf(-8.f, a.x, a.y);
                c.y = fmaf(-8.f, c.x, c.y);
#pragma unroll
                for (int hrow = 0; hrow < 2; ++hrow) {
                    s[j][2 * hrow] = fmaf(s[j][2 * hrow], a.x * ra[hrow], a.y * rb[hrow]);
                    s[j][2 * hrow + 1] = fmaf(s[j][2 * hrow + 1], c.x * ra[hrow], c.y * rb[hrow]);
                }
                if (!plain) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int pos = pos0 + 8 * j + (e ? kb : ka), m = pos - prefix;
                        const bool there = pos < len && ((valid >> (j >> 1)) & 1);
#pragma unroll
                        for (int hrow = 0; hrow < 2; ++hrow) {
                            const bool see = there && (m < 0 || ((s_seen[g + 8 * hrow][m >> 5] >> (m & 31)) & 1u));
                            if (!see) s[j][2 * hrow + e] = -INFINITY;
                        }
                    }
                }
#pragma unroll
                for (int hrow = 0; hrow < 2; ++hrow) most[hrow] = max3(most[hrow], s[j][2 * hrow], s[j][2 * hrow + 1]);
                vs[j] = make_float2(x.x, y.x);
                vm[j] = make_float2(x.y, y.y);
                big = max3(big, x.x, y.x);
            }
#pragma unroll
            for (int q = 1; q < 4; q <<= 1) {
                most[0] = fmaxf(most[0], __shfl_xor_sync(0xffffffffu, most[0], q));
                most[1] = fmaxf(most[1], __shfl_xor_sync(0xffffffffu, most[1], q));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, q));
            }
            const int need = static_cast<int>(__float_as_uint(big) >> 23) - 126;   // 2^need > big
            const bool move = most[0] > top[0] + kNarrowSlack || most[1] > top[1] + kNarrowSlack ||
                              (top[0] == -INFINITY && most[0] > -INFINITY) || (top[1] == -INFINITY && most[1] > -INFINITY) ||
                              (big > 0.f && need > expo);
            if (__any_sync(0xffffffffu, move)) {
                const int was = expo;
                if (big > 0.f) expo = max(expo, need);
                const float unit = exp2i(static_cast<float>(was - expo));
                float f[2];
#pragma unroll
                for (int hrow = 0; hrow < 2; ++hrow) {
                    const float now = fmaxf(top[hrow], most[hrow]);
                    f[hrow] = top[hrow] == -INFINITY ? 0.f : ex2f(top[hrow] - now);
                    top[hrow] = now;
                    sum[hrow] *= f[hrow];
                    mids[hrow] *= f[hrow];
                    f[hrow] *= unit;
                    ones[2 * hrow] *= f[hrow];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) { o[n][0] *= f[0]; o[n][1] *= f[0]; o[n][2] *= f[1]; o[n][3] *= f[1]; }
            }
            const float unit = exp2i(static_cast<float>(-expo));
            const float base[2] = {top[0] == -INFINITY ? 0.f : top[0], top[1] == -INFINITY ? 0.f : top[1]};
            uint32_t pw[4][2];                      // weights of a tile, two keys packed, per row
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float vx = vs[j].x * unit, vy = vs[j].y * unit;
#pragma unroll
                for (int hrow = 0; hrow < 2; ++hrow) {
                    const float px = ex2f(s[j][2 * hrow] - base[hrow]), py = ex2f(s[j][2 * hrow + 1] - base[hrow]);
                    sum[hrow] += px + py;
                    if (plain) {
                        mids[hrow] = fmaf(px, vm[j].x, fmaf(py, vm[j].y, mids[hrow]));
                        pw[j][hrow] = half2_bits(px * vx, py * vy);
                    } else {                        // an unseen key's parameters may be anything
                        const bool sx = s[j][2 * hrow] != -INFINITY, sy = s[j][2 * hrow + 1] != -INFINITY;
                        if (sx) mids[hrow] = fmaf(px, vm[j].x, mids[hrow]);
                        if (sy) mids[hrow] = fmaf(py, vm[j].y, mids[hrow]);
                        pw[j][hrow] = half2_bits(sx ? px * vx : 0.f, sy ? py * vy : 0.f);
                    }
                }
            }
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {        // sixteen keys: tiles 2 jj and 2 jj + 1
                const uint32_t a[4] = {pw[2 * jj][0], pw[2 * jj][1], pw[2 * jj + 1][0], pw[2 * jj + 1][1]};
                mma_f16(ones, a, 0x3c003c00u, 0x3c003c00u);
                const unsigned char *base_v = stage + kNarrowKeys * RB + 16 * jj * RB;
                const int rows[4] = {ka, kb, 8 + ka, 8 + kb};
                uint32_t w[4][NT / 8];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (D == 128) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(base_v + rows[q] * RB + swizzle(rows[q], g >> 1) * 16 + (g & 1) * 8);
                        w[q][0] = v.x; w[q][NT / 8 - 1] = v.y;
                    } else {
                        w[q][0] = *reinterpret_cast<const uint32_t *>(base_v + rows[q] * RB + g * 4);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT / 8; ++n)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const uint32_t x0 = __byte_perm(w[0][n], w[1][n], hf ? 0x7632 : 0x5410);
                        const uint32_t x1 = __byte_perm(w[2][n], w[3][n], hf ? 0x7632 : 0x5410);
                        float(*to)[4] = &o[8 * n + 4 * hf];
                        mma_f16(to[0], a, x0 & 0x000f000fu, x1 & 0x000f000fu);
                        mma_f16(to[1], a, x0 & 0x00f000f0u, x1 & 0x00f000f0u);
                        mma_f16(to[2], a, (x0 >> 8) & 0x000f000fu, (x1 >> 8) & 0x000f000fu);
                        mma_f16(to[3], a, (x0 >> 8) & 0x00f000f0u, (x1 >> 8) & 0x00f000f0u);
                    }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
        for (int q = 1; q < 4; q <<= 1)
#pragma unroll
            for (int hrow = 0; hrow < 2; ++hrow) {
                sum[hrow] += __shfl_xor_sync(0xffffffffu, sum[hrow], q);
                mids[hrow] += __shfl_xor_sync(0xffffffffu, mids[hrow], q);
            }
        __syncwarp();
        // this warp's result as numbers, into its own ring: lane (g, t) holds numbers D / 4 t .. of rows g and g + 8
        float *s_out = reinterpret_cast<float *>(ring);
        const float unit = exp2i(static_cast<float>(expo));
#pragma unroll
        for (int hrow = 0; hrow < 2; ++hrow) {
            float *dst = s_out + (g + 8 * hrow) * D + t * (D / 4);
            const float fixed = fmaf(-8.f * unit, ones[2 * hrow], mids[hrow]);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int n = 0; n < NT / 8; ++n)
#pragma unroll
                    for (int x = 0; x < 8; x += 4) {
                        float4 v;
                        v.x = fmaf(o[8 * n + x][2 * hrow + c], unit * 16777216.f, fixed);
                        v.y = fmaf(o[8 * n + x + 1][2 * hrow + c], unit * 1048576.f, fixed);
                        v.z = fmaf(o[8 * n + x + 2][2 * hrow + c], unit * 16777216.f, fixed);
                        v.w = fmaf(o[8 * n + x + 3][2 * hrow + c], unit * 1048576.f, fixed);
                        *reinterpret_cast<float4 *>(dst + (c * (NT / 8) + n) * 8 + x) = v;
                    }
            if (t == 0) { s_top[warp][g + 8 * hrow] = top[hrow]; s_sum[warp][g + 8 * hrow] = sum[hrow]; }
        }
        __syncthreads();
        // the four warps' results joined: D / 4 threads a row, four numbers each
        const int slot = 2 * blockIdx.x + (k0 > 0 ? 0 : 1);
        float *part = P.part + static_cast<long long>(slot) * kPartFloats<D>;
        for (int x = tid; x < kNarrowRows * (D / 4); x += kNarrowWarps * 32) {
            const int r = x / (D / 4), c = (x % (D / 4)) * 4;
            if (row0 + r >= P.n_rows) break;
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kNarrowWarps; ++w) m = fmaxf(m, s_top[w][r]);
            float l = 0.f;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kNarrowWarps; ++w) {
                // (a warp without a finite or NaN maximum has nothing; a NaN sum stays one)
                const float f = s_top[w][r] == -INFINITY ? (s_sum[w][r] == 0.f ? 0.f : 1.f) : ex2f(s_top[w][r] - m);
                if (f == 0.f) continue;
                const float4 v = *reinterpret_cast<const float4 *>(s_ring + w * kNarrowStages * kNarrowStageBytes<D> + (r * D + c) * 4);
                l = fmaf(f, s_sum[w][r], l);
                a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
            }
            if (whole) {
                const int row = row0 + r, node = row / P.group, h = head * P.group + (row - node * P.group);
                const long long at = b * P.o_seq + node * P.o_node + h * P.o_head + c;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                store_elem<DT>(P.out, at, a.x * inv);
                store_elem<DT>(P.out, at + 1, a.y * inv);
                store_elem<DT>(P.out, at + 2, a.z * inv);
                store_elem<DT>(P.out, at + 3, a.w * inv);
                if (P.lse && c == 0)
                    P.lse[(static_cast<long long>(b) * P.n_nodes + node) * P.n_heads + h] =
                        l == 0.f ? -INFINITY : (m == -INFINITY ? l : (m + log2f(l)) * 0.6931471805599453f);
            } else {
                *reinterpret_cast<float4 *>(part + r * D + c) = a;
                if (c == 0) { part[kNarrowRows * D + r] = m; part[kNarrowRows * (D + 1) + r] = l; }
            }
        }
        u += k1 - k0;
        cur.at += k1 - k0;
        if (u < u_end && cur.at >= static_cast<long long>(cur.units) * items) cur = att_find(P, u, items, lane);
    }
}

// Joins the partial results of items that the cut divided: one CTA per item, which finds the CTAs that
// worked on it from the same arithmetic.
template <int DT, int D>
__global__ void __launch_bounds__(128)
join_kernel(const __grid_constant__ AttendParams P)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int items = P.c.n_heads * P.n_blocks;
    const int b = blockIdx.x / items, item = blockIdx.x - b * items;
    const int len = att_len(P, b), units = att_units(len);
    const long long total = att_units_before(P, P.batch, lane) * items;
    const long long per = max((total + P.n_ctas - 1) / P.n_ctas, 1LL);
    const long long u0 = att_units_before(P, b, lane) * items + static_cast<long long>(item) * units;
    const int first = static_cast<int>(u0 / per), last = static_cast<int>((u0 + units - 1) / per);
    asm volatile("griddepcontrol.wait;" ::: "memory");   // (every thread: this kernel must not end before the one it follows)
    if (units == 0 || first == last) return;
    const int head = item / P.n_blocks, row0 = (item - head * P.n_blocks) * kNarrowRows;
    auto part_of = [&](int cta) { return P.part + static_cast<long long>(2 * cta + (cta == first ? 1 : 0)) * kPartFloats<D>; };
    for (int x = tid; x < kNarrowRows * (D / 4); x += 128) {
        const int r = x / (D / 4), c = (x % (D / 4)) * 4;
        if (row0 + r >= P.n_rows) break;
        float m = -INFINITY;
        for (int k = first; k <= last; ++k) m = fmaxf(m, __ldcg(part_of(k) + kNarrowRows * D + r));
        float l = 0.f;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = first; k <= last; ++k) {
            const float *part = part_of(k);
            const float mk = __ldcg(part + kNarrowRows * D + r), lk = __ldcg(part + kNarrowRows * (D + 1) + r);
            const float f = mk == -INFINITY ? (lk == 0.f ? 0.f : 1.f) : ex2f(mk - m);
            if (f == 0.f) continue;
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + r * D + c));
            l = fmaf(f, lk, l);
            a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
        }
        const int row = row0 + r, node = row / P.group, h = head * P.group + (row - node * P.group);
        const long long at = b * P.o_seq + node * P.o_node + h * P.o_head + c;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        store_elem<DT>(P.out, at, a.x * inv);
        store_elem<DT>(P.out, at + 1, a.y * inv);
        store_elem<DT>(P.out, at + 2, a.z * inv);
        store_elem<DT>(P.out, at + 3, a.w * inv);
        if (P.lse && c == 0)
            P.lse[(static_cast<long long>(b) * P.n_nodes + node) * P.n_heads + h] =
                l == 0.f ? -INFINITY : (m == -INFINITY ? l : (m + log2f(l)) * 0.6931471805599453f);
    }
}

}  // namespace mcsd
