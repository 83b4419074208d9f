// The attention weight that cached rows gather of a chunk's tokens: a key's share of every row that sees it, summed per key head.
#pragma once

#include "mcsd_chunk.cuh"
#include "mcsd_chunk_wide.cuh"

namespace mcsd {

#define MCSD_INLINE __attribute__((always_inline))

// Tokens of sequence b whose weights count: the row of the first one, how many, its position; the rows held before the chunk
// (their weights go on) and with it.
struct WeighSeq { int row, count, pos, old, len; };
__device__ __forceinline__ WeighSeq weigh_seq(const ChunkParams &P, int b)
{
    const ChunkSeq s = chunk_seq(P, b);
    const int skip = P.last > 0 ? max(s.count - P.last, 0) : 0;
    WeighSeq w;
    w.row = s.row + skip;
    w.count = s.count - skip;
    w.old = s.start;
    w.pos = static_cast<int>(min(static_cast<long long>(s.start) + skip, static_cast<long long>(s.len)));     // (none of the rest is there then)
    w.len = s.len;
    return w;
}

// ---- the cut of the work
// An item is a (sequence, key/value head), its units kAttUnit keys each with all rows that see them; a unit has `cost` places
// of the cut, an item `lead` more. As for the attention, all items are cut into runs of equal length, one per CTA, and a unit belongs to the run that
// holds its first place; here nothing has to be joined.
struct WeighItem { int b, head, k0, k1; WeighSeq s; };
struct WeighWalk {
    ChunkPlace left, at, places;                    // of the run; the place in the item, and the item's
    int b, head, units, cost;
    bool fresh;
    // Units and places of one item of sequence b.
    static __device__ __forceinline__ ChunkPlace sizes(const ChunkParams &P, int b, int &units, int &cost)
    {
        const WeighSeq s = weigh_seq(P, b);
        const long long rows = static_cast<long long>(s.count) * P.group;
        units = s.count == 0 || rows < P.least || rows > P.most ? 0 : (s.len + kAttUnit - 1) / kAttUnit;
        cost = 64 + static_cast<int>(min(rows, 1ll << 24));
        return units == 0 ? 0 : static_cast<ChunkPlace>(units) * cost + P.lead;
    }
    __device__ __forceinline__ bool begin(const ChunkParams &P, int lane)
    {
        int u, c;
        const ChunkPlace heads = static_cast<ChunkPlace>(P.c.n_heads);
        ChunkPlace span = 0;
        for (int i = lane; i < P.batch; i += 32) span += sizes(P, i, u, c);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) span += __shfl_xor_sync(0xffffffffu, span, o);
        span *= heads;
        const ChunkPlace per = (span + P.n_ctas - 1) / P.n_ctas;
        ChunkPlace x = blockIdx.x * per;
        if (x >= span) return false;
        left = span - x < per ? span - x : per;
        for (int b0 = 0;; b0 += 32) {
            const ChunkPlace n = b0 + lane < P.batch ? sizes(P, b0 + lane, u, c) * heads : 0;
            ChunkPlace incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const ChunkPlace up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            const unsigned past = __ballot_sync(0xffffffffu, incl > x);
            if (past || b0 + 32 >= P.batch) {
                const int who = past ? __ffs(past) - 1 : 31;
                b = b0 + who;
                x -= __shfl_sync(0xffffffffu, incl - n, who);
                break;
            }
            x -= __shfl_sync(0xffffffffu, incl, 31);
        }
        places = sizes(P, b, units, cost);
        head = static_cast<int>(x / places);
        at = x - head * places;
        fresh = true;
        return true;
    }
    __device__ __forceinline__ bool next(const ChunkParams &P, WeighItem &it)
    {
        for (;;) {
            if (!fresh) {
                if (left <= places - at) return false;
                left -= places - at;
                at = 0;
                if (++head >= P.c.n_heads) {
                    head = 0;
                    do { if (++b >= P.batch) return false; } while ((places = sizes(P, b, units, cost)) == 0);
                }
            }
            fresh = false;
            const ChunkPlace to = at + (left < places - at ? left : places - at);
            auto below = [&](ChunkPlace x) {
                const ChunkPlace k = x <= static_cast<ChunkPlace>(P.lead) ? 0 : (x - P.lead + cost - 1) / cost;
                return k < static_cast<ChunkPlace>(units) ? static_cast<int>(k) : units;
            };
            it.k0 = below(at);
            it.k1 = below(to);
            if (it.k0 >= it.k1) continue;
            it.b = b;
            it.head = head;
            it.s = weigh_seq(P, b);
            return true;
        }
    }
};

// ---- few rows: warp-level matrix instructions, as in the narrow attention kernel
template <int D> constexpr int kWeighStage = kNarrowKeys * (D / 2 + 4);
constexpr int kWeighStages = 4;
template <int D> constexpr int kWeighSmem = kNarrowWarps * kWeighStages * kWeighStage<D>;
template <int NB> constexpr int kWeighCtas = NB == 1 ? 6 : NB == 2 ? 4 : 3;         // per SM

// The first half of the narrow attention kernel (see there): a warp takes every fourth chunk of 32 keys, codes become operands by
// a shift and an AND for two, S^T = K Q^T. A lane then has the scores of four keys with its rows: their weights 2^(s - lse) are added up over its rows
// and, by two shuffles, over the four lanes that share the keys; a key's old weight is on its way meanwhile. No row has a maximum or a sum of its
// own here, so nothing is joined.
// Bytes that must move: key codes, scale and mid, weights read and written. 32 sequences of one token over 4001 rows at most, 8 key heads of 128, 4 query heads each: 25 us
// against 7.6 for the bytes. A CTA has few chunks (about 10 a warp), so that the way to its first one (lengths, pages, codes: 8000 to 20000 cycles
// from launch) and then the issue rate (2000 cycles a chunk and warp with six CTAs an SM) bound it; chunks four ahead, all first loads side by side: 40 -> 25.
template <int DT, int D, int NB>
__global__ void __launch_bounds__(kNarrowWarps * 32, kWeighCtas<NB>)
weigh_narrow_kernel(const __grid_constant__ ChunkParams P)
{
    constexpr int KS = D / 16, JW = D / 32, RB = D / 2, STAGES = kWeighStages, STAGE = kWeighStage<D>;
    extern __shared__ __align__(128) unsigned char s_ring[];
    __shared__ int2 s_pages[kNarrowWarps][STAGES];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int ps = 1 << P.c.page_shift;
    WeighWalk walk;
    if (!walk.begin(P, lane)) return;
    unsigned char *ring = s_ring + warp * STAGES * STAGE;
    auto kappa = [](int c) { return D == 128 ? c ^ ((c >> 1) & 1) : c ^ ((c >> 2) & 1); };
    auto swizzle = [](int row, int chunk) { return D == 128 ? chunk ^ ((row >> 1) & 2) : chunk; };
    const int kg = kappa(g);
    WeighItem it;
    while (walk.next(P, it)) {
        const int k0 = it.k0, k1 = it.k1, len = it.s.len, pos_first = it.s.pos, n_rows = it.s.count * P.group;
        const int left = len - (k0 * kAttUnit + warp * kNarrowKeys);
        const int n_chunks = left <= 0 ? 0 : min(k1 - k0, (left + kAttUnit - 1) / kAttUnit);
        const int32_t *table = P.table + it.b * P.ld_table;
        const unsigned char *pool = P.c.pages + static_cast<long long>(it.head) * kv_block_bytes(D, ps) + lane * 16;
        const int dst_code = smem_u32(ring) + (D == 128 ? (lane >> 2) * RB + swizzle(lane >> 2, lane & 3) * 16 : lane * 16);
        const int dst_param = smem_u32(ring) + kNarrowKeys * RB + (lane & 3) * 16;
        auto page_of = [&](int i) {
            const int pos = (k0 + i) * kAttUnit + warp * kNarrowKeys + (lane & 1) * 16;
            const int page = i < n_chunks && pos < len ? __ldg(table + (pos >> P.c.page_shift)) : -1;
            return static_cast<unsigned>(page) < static_cast<unsigned>(P.c.n_pages) ? page : -1;
        };
        int page_next = -1;
        auto issue = [&](int i, int slot) {
            const int page = page_next;
            if (i < n_chunks) {
                const int row = ((k0 + i) * kAttUnit + warp * kNarrowKeys) & (ps - 1);
                int p[2];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    p[hf] = __shfl_sync(0xffffffffu, page, hf);
                    if (p[hf] >= 0) {
                        const int r = (row + hf * 16) & (ps - 1);
                        const unsigned char *src = pool + p[hf] * P.c.page_stride;
#pragma unroll
                        for (int n = 0; n < D / 64; ++n) cp_async16(dst_code + slot * STAGE + hf * 16 * RB + n * 512, src + r * RB + n * 512);
                        if (lane < 4) cp_async16(dst_param + slot * STAGE + hf * 64, src + ps * D + r * 4);
                    }
                }
                if (lane == 0) s_pages[warp][slot] = make_int2(p[0], p[1]);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        // Pages of the first chunks, queries and lse are asked for before any of them is used.
        int pages[STAGES];
#pragma unroll
        for (int i = 0; i < STAGES; ++i) pages[i] = page_of(i);
        uint4 raw[NB][D / 32];
        float lse[NB][2];
        int token[NB][2];                           // last position that the row sees
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = nb * 8 + g;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) raw[nb][i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < n_rows) {
                const int i = r / P.group, h = it.head * P.group + (r - i * P.group);
                const long long at = (static_cast<long long>(it.s.row) + i) * P.q_token + h * P.q_head + t * (D / 4);
                if (P.q_vec) {
                    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const char *>(P.q) + at * 2);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) raw[nb][i] = __ldg(src + i);
                } else {
                    const unsigned short *src = static_cast<const unsigned short *>(P.q) + at;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
                        raw[nb][i] = make_uint4(src[8 * i] | src[8 * i + 1] << 16, src[8 * i + 2] | src[8 * i + 3] << 16,
                                                src[8 * i + 4] | src[8 * i + 5] << 16, src[8 * i + 6] | src[8 * i + 7] << 16);
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int row = nb * 8 + 2 * t + c;
                float l = INFINITY;
                token[nb][c] = -1;
                if (row < n_rows) {
                    const int i = row / P.group, h = it.head * P.group + (row - i * P.group);
                    l = __ldg(P.lse + (static_cast<long long>(it.s.row) + i) * P.n_heads + h) * 1.4426950408889634f;
                    if (l != -INFINITY) token[nb][c] = pos_first + i;       // (else it counts nothing, whatever its scores are)
                }
                lse[nb][c] = l;
            }
        }
        __syncwarp();                               // (the item before has read its last chunks)
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) {
            page_next = pages[i];
            issue(i, i);
        }
        page_next = pages[STAGES - 1];

        // queries: this lane's D / 4 numbers of row g of every tile, scaled to the top of half's range
        uint32_t qb[NB][KS][2];
        float ra[NB][2], rb[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float x[D / 4];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) Elem<DT>::unpack(raw[nb][i], x + 8 * i);
            float most = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 4; ++i) { most = fmaxf(most, fabsf(x[i])); sum += x[i]; }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            }
            int e = most > 0.f ? static_cast<int>(__float_as_uint(most) >> 23) - 126 : 0;
            e = max(min(e, 112), -110);
            const float up = __int_as_float((127 + 15 - e) << 23);
            const float log2e = P.scale * 1.4426950408889634f;
            const float per_acc = ldexpf(log2e, e - 15 + kKeyExp), per_mid = log2e * sum;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                ra[nb][c] = __shfl_sync(0xffffffffu, per_acc, (2 * t + c) * 4);
                rb[nb][c] = __shfl_sync(0xffffffffu, per_mid, (2 * t + c) * 4);
            }
#pragma unroll
            for (int j = 0; j < JW; ++j)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    qb[nb][2 * j + s][0] = half2_bits(x[8 * j + 2 * s] * up, x[8 * j + 2 * s + 4] * up);
                    qb[nb][2 * j + s][1] = half2_bits(x[8 * j + 2 * s + 1] * up, x[8 * j + 2 * s + 5] * up);
                }
        }

        // this lane's own key of a chunk's 32, for the end: where its weight is (none: null), and what it was
        const int mine = 16 * (t >> 1) + 8 * (t & 1) + kg;
        float *w = nullptr;
        float old = 0.f;
        auto own = [&](int i, int slot) {
            const int pos = (k0 + i) * kAttUnit + warp * kNarrowKeys + mine;
            const int2 pages = s_pages[warp][slot];
            const int page = mine < 16 ? pages.x : pages.y;
            w = i < n_chunks && page >= 0 && pos < len ? P.weights + (static_cast<long long>(page) * P.c.n_heads + it.head) * ps + (pos & (ps - 1)) : nullptr;
            old = w && pos < it.s.old && P.decay != 0.f ? *w : 0.f;
        };
        __syncwarp();
        own(0, 0);
        int slot = 0, fill = STAGES - 1;
        for (int i = 0; i < n_chunks; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();                           // every lane's copies of chunk i are there, and chunk i - 1 is done with
            const unsigned char *stage = ring + slot * STAGE;
            issue(i + STAGES - 1, fill);
            page_next = page_of(i + STAGES);        // (in flight while this chunk is computed)
            const int pos0 = (k0 + i) * kAttUnit + warp * kNarrowKeys;
            float *const to = w;
            const float from = P.decay * old;
            own(i + 1, slot == STAGES - 1 ? 0 : slot + 1);          // (in flight until the next chunk's end)
            const bool plain = pos0 + kNarrowKeys - 1 <= pos_first;
            const __half2 *kp = reinterpret_cast<const __half2 *>(stage + kNarrowKeys * RB);
            float got[2][2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float s[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
                uint32_t v[2][JW];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 16 * m + 8 * x + kg;
                    if constexpr (D == 128) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(stage + row * RB + swizzle(kg, t) * 16);
                        v[x][0] = u.x; v[x][1] = u.y; v[x][2] = u.z; v[x][3] = u.w;
                    } else {
                        const uint2 u = *reinterpret_cast<const uint2 *>(stage + row * RB + t * 8);
                        v[x][0] = u.x; v[x][1] = u.y;
                    }
                }
#pragma unroll
                for (int n = 0; n < JW; ++n) {
                    const uint4 a = key_codes(v[0][n]), c = key_codes(v[1][n]);        // of key kg and of the one eight on
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        mma_f16(s[nb], a.x, c.x, a.y, c.y, qb[nb][2 * n][0], qb[nb][2 * n][1]);
                        mma_f16(s[nb], a.z, c.z, a.w, c.w, qb[nb][2 * n + 1][0], qb[nb][2 * n + 1][1]);
                    }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int key = 16 * m + 8 * x + kg;
                    float2 a = __half22float2(kp[key]);
                    a.y = fmaf(-8.f, a.x, a.y);
                    float sum = 0.f;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float p = ex2f(fmaf(s[nb][2 * x + c], a.x * ra[nb][c], fmaf(a.y, rb[nb][c], -lse[nb][c])));
                            if (plain ? token[nb][c] >= 0 : token[nb][c] >= pos0 + key) sum += p;
                        }
                    got[m][x] = sum;
                }
            }
            float sum = 0.f;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float v = got[m][x];
                    v += __shfl_xor_sync(0xffffffffu, v, 1);
                    v += __shfl_xor_sync(0xffffffffu, v, 2);
                    if (t == 2 * m + x) sum = v;
                }
            if (to) *to = from + sum;
            slot = slot == STAGES - 1 ? 0 : slot + 1;
            fill = fill == STAGES - 1 ? 0 : fill + 1;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
}

// ---- many rows: keys as the rows of tcgen05 products
constexpr int kWeighRows = 256;                     // rows of queries (columns of a product) in a block
constexpr int kWeighKeys = 3;                       // decoded units
constexpr int kWeighAhead = 2;                      // units whose codes are on their way to shared memory
constexpr int kWeighSpread = 12;                    // log2 of what the rows of a block with one scale may lie apart
constexpr int kWeighThreads = 640;                  // 8 warps that add up, 8 that decode, one that issues (and 3 beside it)
template <int D> constexpr int kWeighWideSmem = 1024 + (2 + kWeighKeys) * kWideTile<D> + kWeighKeys * kAttUnit * 8 + kWeighRows * 12 + kWeighAhead * kAttUnit * (D / 2 + 4);

// One CTA per SM. A product has 128 keys as its rows (lanes of tensor memory) and a block of up to 256 rows of queries as its columns, so that a
// thread that adds up has one key: its scale and mid are two registers, its weights are added up without another thread, and what
// differs by column (the sum of a query, its lse) is one broadcast load for two columns. Roles:
//   decoding warps  copy codes two units ahead and turn them into subnormal halves (key_codes), sixteen keys of each unit a warp;
//   issuing warp    S^T = K Q^T into one of two halves of tensor memory, even and odd units in turn;
//   adding groups   even and odd units: 2^(scale_j acc + mid_j rho_n - lse_n), added up over n. Together they bring a block of queries to shared
//                   memory. Where the largest numbers of its rows lie within 2^kWeighSpread of each other, they are scaled by one power of two, and
//                   a factor is the same for all columns: the largest number of a row that is 2^12 below the loudest is at 2^2 at least, and what half's
//                   range takes of its numbers is 2^-25 at most, 2^-27 of that one. Otherwise (a loud row, one that is infinite, one without an lse)
//                   each row has its own, and a column a factor of its own: one more multiplication a score, so that no row takes bits from its neighbours.
// Sequences with more rows than a block take the units once for every block; a key's sum then goes on from what its thread wrote before.
// Of the products only half a softmax is left: one multiply-add, one exponential and one addition per score, in pairs where there is such an instruction.
// 2 x 1500 tokens over 2500 rows, 16 heads of 64: 88 us (floor 11 by the products), 124 with rows far apart in every block; 8 windows of 32 tokens over 3500
// rows, 4 heads to a key head: 27 and 32 (3.7 by the products); 2048 tokens over 8000, 32 heads on 8 of 128: 432. Bound by a group's way through a unit (read the scores, weights, wait: 6300 cycles per 128 x 256), the
// products are done in a third of it.
template <int DT, int D>
__global__ void __launch_bounds__(kWeighThreads, 1)
weigh_wide_kernel(const __grid_constant__ ChunkParams P)
{
    constexpr int TILE = kWideTile<D>, RB = D / 2;
    constexpr uint32_t kColumns = 512;
    extern __shared__ unsigned char s_raw[];
    __shared__ __align__(8) unsigned long long s_bar[2 * kWeighKeys + 6];
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead, s_any;
    __shared__ int s_high[8], s_low[8];             // of a warp's rows: exponents of the largest number of the loudest row, and of the softest
    __shared__ WeighWalk s_walk[kWeighThreads / 32];
    __shared__ WeighItem s_item[kWeighThreads / 32];

    unsigned char *base = s_raw + ((1024 - (smem_u32(s_raw) & 1023)) & 1023);
    unsigned char *s_q = base, *s_k = base + 2 * TILE;                          // [2 x 128 rows], [stages][128 keys]
    float2 *s_param = reinterpret_cast<float2 *>(base + (2 + kWeighKeys) * TILE);       // [stages][keys]{scale, mid - 8 scale}
    float *s_col = reinterpret_cast<float *>(s_param + kWeighKeys * kAttUnit);          // [128 pairs of columns]{rho, rho, lse, lse}
    float *s_factor = s_col + 2 * kWeighRows;                                   // [columns] of a block whose rows lie far apart
    unsigned char *s_codes = reinterpret_cast<unsigned char *>(s_factor + kWeighRows);  // [decoding warps][kWeighAhead]{codes, parameters}

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = smem_u32(s_bar);
    const uint32_t b_full = bars, b_empty = bars + 8 * kWeighKeys, b_s = b_empty + 8 * kWeighKeys, b_read = b_s + 16, b_ready = b_s + 32, b_end = b_s + 40;
    if (tid == 0) {
        for (int i = 0; i < kWeighKeys; ++i) {
            mbar_init(b_full + 8 * i, 8);
            mbar_init(b_empty + 8 * i, 5);          // the products, and the four warps that read the parameters
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_read + 8 * i, 4);
        }
        mbar_init(b_ready, 8 + P.test_extra);       // (0 but in a test of the expiry path: arrivals that never come)
        mbar_init(b_end, 1);
        fence_mbar_init();
        s_dead = 0;
    }
    if (warp == 16) tmem_alloc(smem_u32(&s_tmem), kColumns);
    if (warp == 17) {
        WeighWalk walk;
        const bool any = walk.begin(P, lane);
        if (lane == 0) s_any = any;
        if (any && lane < kWeighThreads / 32) s_walk[lane] = walk;
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    constexpr uint32_t tmem = 0;
    volatile int *dead = &s_dead;
    if (s_tmem != tmem) *dead = 1;                  // (cannot be: all columns are this CTA's)
    const int ps = 1 << P.c.page_shift;
    const int tokens = kWeighRows / P.group;        // of a block

    // Every role goes over the same (block of queries, unit) pairs: f(item, first token, tokens of the block, first and last unit).
    auto for_blocks = [&](auto f) MCSD_INLINE {
        if (!s_any) return;
        for (;;) {
            int more = 0;
            __syncwarp();
            if (lane == 0) more = s_walk[warp].next(P, s_item[warp]);
            if (!__shfl_sync(0xffffffffu, more, 0)) break;
            __syncwarp();
            const WeighItem &it = s_item[warp];
            for (int i0 = 0; i0 < it.s.count; i0 += tokens) {
                const int n = min(tokens, it.s.count - i0);
                // (a block sees nothing behind its last token; the last block sees all units, so that every key gets a number)
                const long long end = (static_cast<long long>(it.s.pos) + i0 + n - 1) / kAttUnit + 1;
                const int k1 = static_cast<int>(min(static_cast<long long>(it.k1), end));
                if (it.k0 < k1) f(it, i0, n, it.k0, k1);
            }
        }
    };

    if (warp >= 8 && warp < 16) {
        // ------------------------------------------------------------ decoding
        regs_down<56>();
        constexpr int CH = RB / 16;                 // 16-byte chunks of a row: 2 or 4; a lane has CH / 2 of those of sixteen keys
        const int key0 = (warp & 7) * 16, c = lane % CH;
        unsigned char *ring = s_codes + (warp & 7) * kWeighAhead * 16 * (RB + 4);
        int stage = 0;
        uint32_t phase = 1;                         // (the first round of stages is free)
        for_blocks([&](const WeighItem &it, int, int, int k0, int k1) MCSD_INLINE {
            const int len = it.s.len;
            const int32_t *table = P.table + it.b * P.ld_table;
            const unsigned char *pool = P.c.pages + static_cast<long long>(it.head) * kv_block_bytes(D, ps);
            auto page_of = [&](int k) MCSD_INLINE {
                const int pos = k * kAttUnit + key0;
                return k < k1 && pos < len ? __ldg(table + (pos >> P.c.page_shift)) : -1;
            };
            uint32_t there = 0u;                    // bit `slot`: the page of that unit's sixteen keys is in the cache
            int page = -1;
            auto issue = [&](int unit, int slot) MCSD_INLINE {
                unsigned char *to = ring + slot * 16 * (RB + 4);
                const bool ok = unit < k1 && static_cast<unsigned>(page) < static_cast<unsigned>(P.c.n_pages);
                there = (there & ~(1u << slot)) | static_cast<uint32_t>(ok) << slot;
                if (ok) {
                    const int r = (unit * kAttUnit + key0) & (ps - 1);
                    const unsigned char *src = pool + page * P.c.page_stride;
#pragma unroll
                    for (int i = 0; i < CH / 2; ++i) cp_async16(smem_u32(to + i * 512 + lane * 16), src + r * RB + lane * 16 + 512 * i);
                    if (lane < 16) cp_async4(to + 16 * RB + lane * 4, src + ps * D + (r + lane) * 4);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            int pages[kWeighAhead + 1];
#pragma unroll
            for (int i = 0; i <= kWeighAhead; ++i) pages[i] = page_of(k0 + i);
#pragma unroll
            for (int i = 0; i < kWeighAhead; ++i) {
                page = pages[i];
                issue(k0 + i, i);
            }
            page = pages[kWeighAhead];
            int slot = 0;
            for (int k = k0; k < k1; ++k) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kWeighAhead - 1) : "memory");
                const unsigned char *from = ring + slot * 16 * (RB + 4);
                wide_wait(b_empty + 8 * stage, phase, dead, P.wait_polls);
#pragma unroll
                for (int i = 0; i < CH / 2; ++i) {  // 16 bytes of codes are four 16-byte chunks of operands
                    const int key = key0 + i * (32 / CH) + lane / CH;
                    unsigned char *tile = s_k + stage * TILE + key * 128;
                    // (with four chunks a row, lanes 2 and 3 take their words in another order: no two lanes of eight meet in a bank)
                    const bool turn = CH == 4 && (c & 2);
                    const uint4 v = *reinterpret_cast<const uint4 *>(from + i * 512 + lane * 16);
                    const uint32_t w[4] = {turn ? v.z : v.x, turn ? v.w : v.y, turn ? v.x : v.z, turn ? v.y : v.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int chunk = 4 * c + (turn ? j ^ 2 : j);
                        *reinterpret_cast<uint4 *>(tile + (chunk >> 3) * (kAttUnit * 128) + (((chunk & 7) ^ (key & 7)) << 4)) =
                            key_codes(w[j]);
                    }
                }
                if (lane < 16) {
                    const float2 p = (there >> slot) & 1u ? __half22float2(*reinterpret_cast<const __half2 *>(from + 16 * RB + lane * 4)) : make_float2(0.f, 0.f);
                    s_param[stage * kAttUnit + key0 + lane] = make_float2(p.x, fmaf(-8.f, p.x, p.y));
                }
                fence_proxy_async();
                warp_arrive(b_full + 8 * stage, lane);
                if (++stage == kWeighKeys) { stage = 0; phase ^= 1; }
                issue(k + kWeighAhead, slot);       // (what this lane had there is read)
                page = page_of(k + kWeighAhead + 1);
                slot = slot == kWeighAhead - 1 ? 0 : slot + 1;
            }
        });
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= 16) {
        // ------------------------------------------------------------ issuing
        regs_down<32>();
        if (warp == 16) {
            int stage = 0;
            uint32_t phase = 0, blocks = 0, n[2] = {0, 0};
            const uint32_t q_at = tc_operand(smem_u32(s_q), 16);
            for_blocks([&](const WeighItem &, int, int n_tokens, int k0, int k1) MCSD_INLINE {
                wide_wait(b_ready, blocks & 1, dead, P.wait_polls);
                ++blocks;
                const uint32_t shape = tc_shape((n_tokens * P.group + 63) & ~63, false);
                for (int k = k0; k < k1; ++k) {
                    const int x = k & 1;
                    wide_wait(b_full + 8 * stage, phase, dead, P.wait_polls);
                    const uint32_t m = x ? n[1]++ : n[0]++;
                    if (m > 0) wide_wait(b_read + 8 * x, (m - 1) & 1, dead, P.wait_polls);
                    tc_after_sync();
                    const uint32_t at = tc_operand(smem_u32(s_k) + stage * TILE, 16);
#pragma unroll
                    for (int s = 0; s < D / 16; ++s)
                        tc_mma_ss(tmem + 256 * x, at + (s >> 2) * (kAttUnit * 128 / 16) + (s & 3) * 2, q_at + (s >> 2) * (kWeighRows * 128 / 16) + (s & 3) * 2, kOperandHigh,
                                  shape, s > 0);
                    tc_commit(b_s + 8 * x);
                    tc_commit(b_empty + 8 * stage);
                    if (++stage == kWeighKeys) { stage = 0; phase ^= 1; }
                }
            });
            // (what was issued ends before its memory is given back, whichever wait expired)
            tc_commit(b_end);
            for (uint32_t i = 0; i < kWaitPolls && !__all_sync(0xffffffffu, mbar_try_wait(b_end, 0)); ++i) {}
        }
    } else {
        // ------------------------------------------------------------ adding up
        regs_up<168>();
        const int x = warp >> 2, r = tid & 127;     // group; key of the unit = lane of tensor memory
        const uint32_t t_s = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 256 * x;
        int stage = 0;
        uint32_t phase = 0, n = 0;
        auto both = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
        for_blocks([&](const WeighItem &it, int i0, int n_tokens, int k0, int k1) MCSD_INLINE {
            const int n_rows = n_tokens * P.group, columns = (n_rows + 63) & ~63;
            float factor;                           // log2 units per unit of scale acc + (mid - 8 scale) rho: of all columns, or of this thread's
            bool apart;                             // whether each column has its own
            {
                // queries of the block: row `tid`, in the order that the ANDs of the keys give
                uint4 raw[D / 8];
#pragma unroll
                for (int c = 0; c < D / 8; ++c) raw[c] = make_uint4(0u, 0u, 0u, 0u);
                float lse = INFINITY;               // (of no row: no weight)
                bool none = false;                  // a row without an lse: it counts nothing, whatever its queries and the keys are
                if (tid < n_rows) {
                    const int i = tid / P.group, h = it.head * P.group + (tid - i * P.group);
                    const long long token = static_cast<long long>(it.s.row) + i0 + i, at = token * P.q_token + h * P.q_head;
                    lse = __ldg(P.lse + token * P.n_heads + h) * 1.4426950408889634f;
                    none = lse == -INFINITY;
                    if (none) {                     // (its queries stay zeros)
                    } else if (P.q_vec) {
#pragma unroll
                        for (int c = 0; c < D / 8; ++c) raw[c] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const char *>(P.q) + 2 * at) + c);
                    } else {
                        const unsigned short *src = static_cast<const unsigned short *>(P.q) + at;
#pragma unroll
                        for (int c = 0; c < D / 8; ++c)
                            raw[c] = make_uint4(src[8 * c] | src[8 * c + 1] << 16, src[8 * c + 2] | src[8 * c + 3] << 16,
                                                src[8 * c + 4] | src[8 * c + 5] << 16, src[8 * c + 6] | src[8 * c + 7] << 16);
                    }
                }
                float most = 0.f, sum = 0.f;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    float v[8];
                    Elem<DT>::unpack(raw[c], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) { most = fmaxf(most, fabsf(v[i])); sum += v[i]; }
                }
                int e = most > 0.f ? max(min(static_cast<int>(__float_as_uint(most) >> 23) - 126, 112), -110) : 0;
                int high = __reduce_max_sync(0xffffffffu, most > 0.f ? e : -110), low = __reduce_min_sync(0xffffffffu, none ? -1000 : most > 0.f ? e : 112);
                if (lane == 0) { s_high[warp] = high; s_low[warp] = low; }
                both();                             // (and all scores of the block before are there: its queries are done with)
#pragma unroll
                for (int w = 0; w < 8; ++w) { high = max(high, s_high[w]); low = min(low, s_low[w]); }
                apart = high - low > kWeighSpread;
                if (!apart) e = high;               // (a block of zeros: any)
                const float up = __int_as_float((127 + 15 - e) << 23);
                factor = ldexpf(P.scale * 1.4426950408889634f, e - 15 + kKeyExp);
                s_factor[tid] = none ? __int_as_float(0x7fffffff) : factor;      // (NaN: the column's weights are dropped)
                s_col[(tid >> 1) * 4 + (tid & 1)] = sum * up * kKeyUnit;
                s_col[(tid >> 1) * 4 + 2 + (tid & 1)] = lse;
                unsigned char *to = s_q + tid * 128;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    float v[8];
                    Elem<DT>::unpack(raw[c], v);
                    uint32_t out[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[i] = half2_bits(v[i] * up, v[i + 4] * up);
                    *reinterpret_cast<uint4 *>(to + (c >> 3) * (kWeighRows * 128) + (((c & 7) ^ (tid & 7)) << 4)) = make_uint4(out[0], out[1], out[2], out[3]);
                }
                fence_proxy_async();
                both();                             // (the columns' numbers are there)
                warp_arrive(b_ready, lane);
            }
            const int32_t *table = P.table + it.b * P.ld_table;
            const long long first = static_cast<long long>(it.s.pos) + i0;      // position of the block's first token
            const int len = it.s.len;
            auto page_of = [&](int k) MCSD_INLINE { return k < k1 && k * kAttUnit + r < len ? __ldg(table + ((k * kAttUnit + r) >> P.c.page_shift)) : -1; };
            int page_next = page_of((k0 & 1) == x ? k0 : k0 + 1);
            for (int k = k0; k < k1; ++k) {
                if ((k & 1) == x) {
                    // where this key's weight lies, and what it starts from
                    const int pos = k * kAttUnit + r, page = page_next;
                    page_next = page_of(k + 2);
                    const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(P.c.n_pages);
                    float *w = P.weights + (static_cast<long long>(there ? page : 0) * P.c.n_heads + it.head) * ps + (pos & (ps - 1));
                    float old = 0.f;
                    // (a block goes on from the one before where that has seen the unit, too)
                    if (there && i0 > 0 && static_cast<long long>(k) * kAttUnit < first) old = *w;
                    else if (there && pos < it.s.old && P.decay != 0.f) old = P.decay * *w;
                    wide_wait(b_full + 8 * stage, phase, dead, P.wait_polls);
                    const float2 par = s_param[stage * kAttUnit + r];
                    warp_arrive(b_empty + 8 * stage, lane);
                    const float2 a = make_float2(par.x * factor, par.x * factor), m = make_float2(par.y * factor, par.y * factor);
                    wide_wait(b_s + 8 * x, n & 1, dead, P.wait_polls);
                    ++n;
                    tc_after_sync();
                    float2 s0 = make_float2(0.f, 0.f), s1 = make_float2(0.f, 0.f);
                    // plain: all columns see the key; even: they have one factor; from: first column that sees the key
                    auto add = [&](auto plain_tag, auto even_tag, int from) MCSD_INLINE {
                        constexpr bool plain = decltype(plain_tag)::value, even = decltype(even_tag)::value;
#pragma unroll 1
                        for (int c = 0; c < columns; c += 64) {
                            uint32_t acc[64];
                            tmem_load64(t_s + c, acc);
                            const float4 *col = reinterpret_cast<const float4 *>(s_col) + (c >> 1);
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                const float4 v = col[j];
                                const float2 got = make_float2(__uint_as_float(acc[2 * j]), __uint_as_float(acc[2 * j + 1])), rho = make_float2(v.x, v.y),
                                             less = make_float2(-v.z, -v.w);
                                float2 e, f;
                                if constexpr (even) {
                                    e = fma2(a, got, fma2(m, rho, less));
                                } else {
                                    f = *reinterpret_cast<const float2 *>(s_factor + c + 2 * j);
                                    e = fma2(fma2(make_float2(par.x, par.x), got, __fmul2_rn(make_float2(par.y, par.y), rho)), f, less);
                                }
                                float2 p = make_float2(ex2f(e.x), ex2f(e.y));
                                if (!plain) {
                                    if (c + 2 * j < from || c + 2 * j >= n_rows) p.x = 0.f;
                                    if (c + 2 * j + 1 < from || c + 2 * j + 1 >= n_rows) p.y = 0.f;
                                }
                                if constexpr (!even) {
                                    if (f.x != f.x) p.x = 0.f;
                                    if (f.y != f.y) p.y = 0.f;
                                }
                                if (j & 1) s1 = add2(s1, p); else s0 = add2(s0, p);
                            }
                        }
                    };
                    if (!apart && (k + 1) * static_cast<long long>(kAttUnit) - 1 <= first) {
                        add(std::true_type(), std::true_type(), 0);
                    } else {
                        const long long token = pos - first;
                        const int from = token <= 0 ? 0 : static_cast<int>(min(token * P.group, 1ll << 20));
                        if (apart) add(std::false_type(), std::false_type(), from);
                        else add(std::false_type(), std::true_type(), from);
                    }
                    tc_before_sync();
                    warp_arrive(b_read + 8 * x, lane);
                    const float sum = (s0.x + s0.y) + (s1.x + s1.y);
                    if (there) *w = *dead ? __int_as_float(0x7fffffff) : old + sum;
                }
                if (++stage == kWeighKeys) { stage = 0; phase ^= 1; }
            }
        });
    }
    tc_before_sync();
    __syncthreads();
    if (warp == 16) {
        tc_after_sync();
        tmem_free(tmem, kColumns);
    }
}

#undef MCSD_INLINE

}  // namespace mcsd
