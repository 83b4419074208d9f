// Attention of a flattened draft tree over the paged 4-bit cache.
#pragma once

#include <type_traits>

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
    uint32_t lead;                                  // places of the cut an item costs beside its units
    int32_t q_vec, o_vec;                           // rows of q may be read, those of out written in 16-byte vectors
    float scale;
    float scale_part;                               // |scale| log2(e) = scale_part 2^scale_power, the part below 1
    int32_t scale_power;
    uint32_t wait_polls;                            // poll budget of the bounded waits (kWaitPolls unless a test shortens it)
    uint32_t test_extra;                            // 0; a test of the expiry path has a barrier wait for this many more arrivals
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

// The cut: `span` places in all, `per` of them to a CTA. An item begins with `lead` places that stand for what it costs
// beside its units (its queries, the units that hold the tree, its results). Without them a CTA with many short
// items is the last to end: 32 sequences of up to 1000 positions, 31 rows x 32 heads: 249 -> 126 us; 4 of up to 16001, 724 rows
// x 8 heads: 294 -> 171 us; 64 decoding ones of up to 8191 x 8 heads: 103 -> 87 us (random lengths; equal ones are as before).
struct AttCut { uint32_t lead, span, per; };

// Places before sequence `stop` (all of them for stop == batch) of one item per sequence; every lane gets the sum.
// (The host refuses calls that could have 2^32 places in all.)
__device__ __forceinline__ uint32_t att_before(const AttendParams &P, uint32_t lead, int stop, int lane)
{
    uint32_t sum = 0;
    for (int b = lane; b < stop; b += 32) {
        const int len = att_len(P, b);
        if (len >= 0) sum += static_cast<uint32_t>(att_units(len)) + lead;
    }
    return __reduce_add_sync(0xffffffffu, sum);
}
__device__ __forceinline__ AttCut att_cut(const AttendParams &P, uint32_t items, int lane)
{
    AttCut cut;
    uint32_t sum = 0, used = 0;
    for (int b = lane; b < P.batch; b += 32) {
        const int len = att_len(P, b);
        sum += static_cast<uint32_t>(att_units(len));
        used += len >= 0;
    }
    sum = __reduce_add_sync(0xffffffffu, sum) * items;
    used = __reduce_add_sync(0xffffffffu, used) * items;
    const uint32_t n = static_cast<uint32_t>(P.n_ctas);
    cut.lead = sum > n ? P.lead : 0u;                // (otherwise every unit has a CTA of its own)
    cut.span = sum + cut.lead * used;
    cut.per = max(cut.span / n + (cut.span % n != 0u), 1u);
    return cut;
}

// Position in the cut: a sequence, its length and places per item, and the place within its items.
struct AttCursor { int b, len; uint32_t places, at; };

// The sequence that holds place `u` (of all items); u must be below the span.
__device__ __forceinline__ AttCursor att_find(const AttendParams &P, const AttCut &cut, uint32_t u, uint32_t items, int lane)
{
    AttCursor c;
    uint32_t before = 0;
    for (int b0 = 0;; b0 += 32) {
        const int b = b0 + lane;
        const int len = b < P.batch ? att_len(P, b) : -1;
        const uint32_t n = len < 0 ? 0u : static_cast<uint32_t>(att_units(len)) + cut.lead;
        uint32_t incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        const unsigned past = __ballot_sync(0xffffffffu, (before + incl) * items > u);
        if (past || b0 + 32 >= P.batch) {
            const int who = past ? __ffs(past) - 1 : 31;
            c.b = b0 + who;
            c.places = __shfl_sync(0xffffffffu, n, who);
            c.len = __shfl_sync(0xffffffffu, len, who);
            c.at = u - (before + __shfl_sync(0xffffffffu, incl - n, who)) * items;
            return c;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
}

// What a CTA has of the item its cursor stands in: units [k0, k1) of `units`, `places` of the cut in all; k1 <= 0: its
// run ends before the item's first unit (which can only be the last item of a run).
struct AttPiece { int item, units, k0, k1; uint32_t places; };
__device__ __forceinline__ AttPiece att_piece(const AttCut &cut, const AttCursor &cur, uint32_t left)
{
    AttPiece x;
    x.item = static_cast<int>(cur.at / cur.places);
    const uint32_t from = cur.at - static_cast<uint32_t>(x.item) * cur.places;
    x.places = left < cur.places - from ? left : cur.places - from;
    x.units = static_cast<int>(cur.places - cut.lead);
    x.k0 = max(static_cast<int>(from - cut.lead), 0);
    x.k1 = static_cast<int>(from + x.places - cut.lead);
    return x;
}

// ---- few rows: warp-level matrix instructions on codes that go from shared memory to registers
constexpr int kNarrowWarps = 4, kNarrowKeys = 32;
constexpr float kNarrowSlack = 4.f, kNoTop = -3e38f;
constexpr float kLeastLevel = -24.f;                // log2 of the smallest value scale
template <int NB> constexpr int kNarrowRows = 8 * NB;                   // rows of a block
template <int NB> constexpr int kNarrowStages = NB == 1 ? 3 : 4;
template <int NB> constexpr int kNarrowCtas = NB == 1 ? 4 : NB == 2 ? 3 : 2;          // CTAs per SM
template <int D> constexpr int kNarrowStageBytes = kNarrowKeys * (D + 8);
template <int D, int NB> constexpr int kNarrowSmem = kNarrowWarps * kNarrowStages<NB> * kNarrowStageBytes<D>;
// a partial result: rows x D, maxima, sums
__host__ __device__ __forceinline__ constexpr int part_floats(int rows, int dim) { return rows * (dim + 2); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {            // of an 8 x 8 matrix of halves across the warp
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// What a CTA has of an item: units [k0, k1) of one block of rows of one (sequence, key/value head). Rows row0 .. rows - 1 of the head's
// are the block's (or fewer: a block has at most as many as the kernel's), the first `tail` positions are seen by all of them;
// whole: all of the item's units; last (of chunks): the CTA that has the last of them.
struct AttItem { int b, head, len, tail, row0, rows, k0, k1; bool whole; int last; };
// Where a part of an item goes: a CTA has one that others began and one that others end at most.
__device__ __forceinline__ long long att_slot(int k0) { return 2 * blockIdx.x + (k0 > 0 ? 0 : 1); }

// The rows of a tree: those of all nodes, as the narrow kernel and its like see them.
struct TreeRows {
    typedef AttendParams Params;
    struct Walk {
        AttCut cut;
        AttCursor cur;
        uint32_t u, u_end;
        AttPiece piece;
        __device__ __forceinline__ bool begin(const AttendParams &P, int lane)
        {
            const uint32_t items = static_cast<uint32_t>(P.c.n_heads * P.n_blocks);
            cut = att_cut(P, items, lane);
            if (cut.span == 0 || blockIdx.x > (cut.span - 1) / cut.per) return false;      // (runs before the last one are whole)
            u = blockIdx.x * cut.per;
            u_end = cut.span - u < cut.per ? cut.span : u + cut.per;
            cur = att_find(P, cut, u, items, lane);
            return true;
        }
        // What the run has at its place (false: nothing any more), and, behind the work on it, the way to the next place. (Both in one step ahead of
        // the work took more registers: 26.0 -> 27.0 us of 8 sequences x 7 nodes, 32 heads on 8, 36.4 -> 37.8 of 13 nodes, 32 heads.)
        template <int ROWS>
        __device__ __forceinline__ bool here(const AttendParams &P, int, AttItem &it)
        {
            if (u >= u_end) return false;
            piece = att_piece(cut, cur, u_end - u);
            if (piece.k1 <= 0) return false;
            it.b = cur.b;
            it.len = cur.len;
            it.head = piece.item / P.n_blocks;
            it.row0 = (piece.item - it.head * P.n_blocks) * ROWS;
            it.rows = P.n_rows;
            it.tail = P.prefix_len[it.b];
            it.k0 = piece.k0;
            it.k1 = piece.k1;
            it.whole = piece.k0 == 0 && piece.k1 == piece.units;
            return true;
        }
        __device__ __forceinline__ void on(const AttendParams &P, int lane)
        {
            const uint32_t items = static_cast<uint32_t>(P.c.n_heads * P.n_blocks);
            u += piece.places;
            cur.at += piece.places;
            if (u < u_end && cur.at >= cur.places * items) cur = att_find(P, cut, u, items, lane);
        }
    };
    // (the joining kernel finds what was divided by itself)
    static __device__ __forceinline__ void begun(const AttendParams &) {}
    static __device__ __forceinline__ void divided(const AttendParams &, const AttItem &) {}
    static __device__ __forceinline__ long long q_at(const AttendParams &P, const AttItem &it, int row)
    {
        const int node = row / P.group, h = it.head * P.group + (row - node * P.group);
        return it.b * P.q_seq + node * P.q_node + h * P.q_head;
    }
    // Positions behind `tail` that a row sees, a bit each.
    static __device__ __forceinline__ void see(const AttendParams &P, const AttItem &it, int row, uint32_t *seen)
    {
        for (int i = 0; i * 32 < P.n_nodes; ++i) seen[i] = 0u;
        int a = row < it.rows ? row / P.group : -1;
        while (a >= 0) {
            seen[a >> 5] |= 1u << (a & 31);
            a = P.parent[a];
        }
    }
    static __device__ __forceinline__ long long out_at(const AttendParams &P, const AttItem &it, int row)
    {
        const int node = row / P.group, h = it.head * P.group + (row - node * P.group);
        return it.b * P.o_seq + node * P.o_node + h * P.o_head;
    }
    static __device__ __forceinline__ long long lse_at(const AttendParams &P, const AttItem &it, int row)
    {
        const int node = row / P.group;
        return (static_cast<long long>(it.b) * P.n_nodes + node) * P.n_heads + it.head * P.group + (row - node * P.group);
    }
};

// Stores four numbers of a finished row, and its log-sum.
template <int DT, class Rows>
__device__ __forceinline__ void att_store(const typename Rows::Params &P, const AttItem &it, int row, int c, float4 a, float m, float l)
{
    const long long at = Rows::out_at(P, it, row) + c;
    const float inv = l == 0.f ? 0.f : 1.f / l;     // (nothing seen: zeros)
    store_elem<DT>(P.out, at, a.x * inv);
    store_elem<DT>(P.out, at + 1, a.y * inv);
    store_elem<DT>(P.out, at + 2, a.z * inv);
    store_elem<DT>(P.out, at + 3, a.w * inv);
    if (P.lse && c == 0) P.lse[Rows::lse_at(P, it, row)] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}
__device__ __forceinline__ float lg2f(float x) { float r; asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// log2 of a value scale (a row without a range counts as the smallest scale, so that its probability stays in range; what is
// not a scale at all, on a key that nobody sees, as well).
__device__ __forceinline__ float att_level(float scale) { return fmaxf(lg2f(scale), kLeastLevel); }
// Factor that brings a partial result with maximum m and sum l to the maximum `top`; a NaN sum stays one.
__device__ __forceinline__ float att_factor(float m, float l, float top) { return l == l ? ex2f(m - top) : 1.f; }

// Four warps; a warp takes every fourth chunk of 32 keys of the CTA's run with running maxima, sums and
// weighted sums of its own, so that nothing but the end of an item joins them.  Keys are the long side of the
// matrix instructions (S^T = K Q^T, O^T = V^T P^T), so that a block has 8, 16 or 24 rows and decoding wastes little.
//
// The codes never become numbers in memory.  A 4-bit code c in the lowest bits of a half is the subnormal
// number c 2^-24, one in bits 4 to 7 is 16 c 2^-24: one AND turns eight codes of a word into operands of
// the matrix instruction (two at a time), exactly; Q carries the 1/16 of the odd codes, the end of an item that
// of the odd output columns.  With mid and scale of a row,
//   <q, k_j> = scale_j sum q c_j + (mid_j - 8 scale_j) sum q
//   sum_j p_j v_j = sum_j (p_j vscale_j) c_j - 8 sum_j (p_j vscale_j) + sum_j p_j vmid_j
// where p vscale is rounded to half once and both of its sums (the second by a matrix instruction with ones)
// use the rounded weight; scores, maxima, sums and the rest are float32.  Q is scaled by a power of two per row so
// that no type's range matters.  The reference of a row's exponents is the maximum of s_j + log2 vscale_j over the keys
// that the row sees: its largest weight p vscale lies near 1, and half's range costs the others 2^-25 of that one at
// most, whatever scales stand on keys that it does not see or hardly weighs (relative to the largest score and the largest scale
// met, a loud value anywhere takes bits from all rows).  A weight may exceed 1 by 2^kNarrowSlack before the reference is moved,
// so the sums are rescaled seldom and the usual chunk needs one vote instead of reductions.
//
// Measured: 64 sequences of up to 8191 positions, 8 key heads, 4 query heads each: 92 us, 3.9 TB/s of the algorithm's bytes,
// 0.60 of the measured copy bandwidth; 8 sequences of up to 2050 positions x 32 heads, 45 rows: 77 us. The 32-bit logic
// pipe bounds it (53 % busy: an AND for every two codes and row block, a byte permutation and a shift for every
// eight of the values), then the warps' own latencies; with queries as the long side (sixteen rows a block, a
// maximum by shuffles in every chunk) the first took 165 us. Blocks of 24 rows take 255 registers, eight warps per SM; with
// D = 128 every form spills a few words (stored: 16 to 92 bytes a thread over a tree's rows, 12 to 276 over a chunk's).
//
// Row c of a tile of eight keys is key kappa(c): with this order (and, where a row has four 16-byte chunks, those of
// rows 4 to 7 exchanged by two) every shared-memory load of codes touches each bank once.
template <int DT, int D, int NB, class Rows>
__global__ void __launch_bounds__(kNarrowWarps * 32, kNarrowCtas<NB>)
narrow_kernel(const __grid_constant__ typename Rows::Params P)
{
    constexpr int MT = D / 16;                      // m16 tiles of the output
    constexpr int KS = D / 16;                      // k16 steps of the scores
    constexpr int JW = D / 32;                      // words of codes a lane holds of a key row
    constexpr int RB = D / 2;                       // bytes of a code row
    constexpr int ROWS = kNarrowRows<NB>, STAGES = kNarrowStages<NB>, STAGE = kNarrowStageBytes<D>;
    extern __shared__ __align__(128) unsigned char s_ring[];
    __shared__ uint32_t s_seen[ROWS][MCSD_MAX_NODES / 32];
    __shared__ float s_top[kNarrowWarps][ROWS], s_sum[kNarrowWarps][ROWS];
    __shared__ int s_valid[kNarrowWarps][STAGES];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int ps = 1 << P.c.page_shift;
    if (tid == 0) Rows::begun(P);
    typename Rows::Walk walk;
    if (!walk.begin(P, lane)) return;
    AttItem it;
    unsigned char *ring = s_ring + warp * STAGES * STAGE;
    auto kappa = [](int c) { return D == 128 ? c ^ ((c >> 1) & 1) : c ^ ((c >> 2) & 1); };
    auto swizzle = [](int row, int chunk) { return D == 128 ? chunk ^ ((row >> 1) & 2) : chunk; };
    const int kg = kappa(g), ka = kappa(2 * t), kb = kappa(2 * t + 1);

    for (; walk.template here<ROWS>(P, lane, it); walk.on(P, lane)) {
        const int k0 = it.k0, k1 = it.k1, b = it.b, len = it.len, head = it.head, row0 = it.row0, prefix = it.tail;

        __syncthreads();                            // the shared memory of the item before is free
        // this warp's chunks: keys [128 k + 32 warp, + 32) for k = k0 .. k1 - 1, as far as there are keys
        const int left = len - (k0 * kAttUnit + warp * kNarrowKeys);
        const int n_chunks = left <= 0 ? 0 : min(k1 - k0, (left + kAttUnit - 1) / kAttUnit);
        const int32_t *table = P.table + b * P.ld_table;
        const unsigned char *pool = P.c.pages + static_cast<long long>(head) * kv_block_bytes(D, ps) + lane * 16;
        const int v_at = ps * RB;                   // value codes, then the parameters of keys and values
        const int dst_code = smem_u32(ring) + (D == 128 ? (lane >> 2) * RB + swizzle(lane >> 2, lane & 3) * 16 : lane * 16);
        const int p_at = ps * D + (lane >> 2) * ps * 4 + ((lane & 3) - lane) * 16;
        const int dst_param = smem_u32(ring) + kNarrowKeys * D + (lane >> 2) * kNarrowKeys * 4 + (lane & 3) * 16;
        // page of this lane's half (16 keys) of chunk i, -1 where there is none
        auto page_of = [&](int i) {
            const int pos = (k0 + i) * kAttUnit + warp * kNarrowKeys + (lane & 1) * 16;
            return i < n_chunks && pos < len ? __ldg(table + (pos >> P.c.page_shift)) : -1;
        };
        int page_next = page_of(0);
        auto issue = [&](int i, int slot) {
            const int page = page_next;
            page_next = page_of(i + 1);             // (its load is in flight while the next chunk is computed)
            if (i < n_chunks) {
                int ok = 0;
                const int row = (i * kAttUnit + k0 * kAttUnit + warp * kNarrowKeys) & (ps - 1);
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int p = __shfl_sync(0xffffffffu, page, hf);
                    if (static_cast<unsigned>(p) < static_cast<unsigned>(P.c.n_pages)) {
                        ok |= 1 << hf;
                        const int r = (row + hf * 16) & (ps - 1);
                        const unsigned char *src = pool + p * P.c.page_stride;
                        const unsigned char *codes = src + r * RB;
                        const uint32_t to = dst_code + slot * STAGE + hf * 16 * RB;
#pragma unroll
                        for (int n = 0; n < D / 64; ++n) {
                            cp_async16(to + n * 512, codes + n * 512);
                            cp_async16(to + n * 512 + kNarrowKeys * RB, codes + v_at + n * 512);
                        }
                        if (lane < 8) cp_async16(dst_param + slot * STAGE + hf * 64, src + p_at + r * 4);
                    }
                }
                if (lane == 0) s_valid[warp][slot] = ok;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) issue(i, i);

        if (tid < ROWS) Rows::see(P, it, row0 + tid, s_seen[tid]);
        if (tid == 0) Rows::divided(P, it);
        // queries: this lane's D / 4 numbers of row g of every tile, scaled to the top of half's range
        uint32_t qb[NB][KS][2];
        float ra[NB][2], rb[NB][2];                 // of rows 2 t and 2 t + 1: log2 units per unit of an accumulator, and per unit of mid - 8 scale
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = row0 + nb * 8 + g;
            float x[D / 4];
#pragma unroll
            for (int i = 0; i < D / 4; ++i) x[i] = 0.f;
            if (r < it.rows) {
                const long long at = Rows::q_at(P, it, r) + t * (D / 4);
                if (P.q_vec) {
                    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const char *>(P.q) + at * 2);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) Elem<DT>::unpack(src[i], x + 8 * i);   // (not the read-only path: out may be q)
                } else {
#pragma unroll
                    for (int i = 0; i < D / 4; ++i) x[i] = load_elem<DT>(P.q, at + i);
                }
            }
            float most = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 4; ++i) { most = fmaxf(most, fabsf(x[i])); sum += x[i]; }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            }
            // 2^e > most >= 2^(e - 1); the row is scaled by 2^(15 - e)
            int e = most > 0.f ? static_cast<int>(__float_as_uint(most) >> 23) - 126 : 0;
            e = max(min(e, 112), -110);
            const float up = __int_as_float((127 + 15 - e) << 23);
            const float log2e = P.scale * 1.4426950408889634f;
            const float per_acc = ldexpf(log2e, e - 15 + 24), per_mid = log2e * sum;
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
                    qb[nb][2 * j + s][1] = half2_bits(x[8 * j + 2 * s + 1] * up * 0.0625f, x[8 * j + 2 * s + 5] * up * 0.0625f);
                }
        }
        __syncthreads();

        float o[NB][MT][4], ones[NB][4], top[NB][2], sum[NB][2], mids[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int i = 0; i < MT; ++i) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.f;
            ones[nb][0] = ones[nb][1] = ones[nb][2] = ones[nb][3] = 0.f;
            top[nb][0] = top[nb][1] = kNoTop;
            sum[nb][0] = sum[nb][1] = mids[nb][0] = mids[nb][1] = 0.f;
        }

        // One chunk; `plain`: every row sees every key of it.
        auto chunk = [&](auto plain_tag, const unsigned char *stage, int pos0, int valid) {
            constexpr bool plain = decltype(plain_tag)::value;
            float s[NB][2][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int m = 0; m < 2; ++m) s[nb][m][0] = s[nb][m][1] = s[nb][m][2] = s[nb][m][3] = 0.f;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                uint32_t w[2][JW];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 16 * m + 8 * x + kg;
                    if constexpr (D == 128) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(stage + row * RB + swizzle(kg, t) * 16);
                        w[x][0] = v.x; w[x][1] = v.y; w[x][2] = v.z; w[x][3] = v.w;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2 *>(stage + row * RB + t * 8);
                        w[x][0] = v.x; w[x][1] = v.y;
                    }
                }
#pragma unroll
                for (int n = 0; n < JW; ++n) {
                    const uint32_t y0 = w[0][n] >> 8, y1 = w[1][n] >> 8;
                    const uint32_t a[4] = {w[0][n] & 0x000f000fu, w[1][n] & 0x000f000fu, w[0][n] & 0x00f000f0u, w[1][n] & 0x00f000f0u};
                    const uint32_t c[4] = {y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        mma_f16(s[nb][m], a[0], a[1], a[2], a[3], qb[nb][2 * n][0], qb[nb][2 * n][1]);
                        mma_f16(s[nb][m], c[0], c[1], c[2], c[3], qb[nb][2 * n + 1][0], qb[nb][2 * n + 1][1]);
                    }
                }
            }
            const __half2 *kp = reinterpret_cast<const __half2 *>(stage + kNarrowKeys * D);
            const __half2 *vp = kp + kNarrowKeys;
            float vs[2][2], vm[2][2];
            float most[NB][2];                      // largest weight of each row among this lane's keys (-inf: it sees none of them), log2
            // scores in log2 units: element c of tile m is (key 16 m + 8 (c / 2) + kappa(g), row 2 t + c % 2)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int key = 16 * m + 8 * x + kg;
                    float2 a = __half22float2(kp[key]), v = __half22float2(vp[key]);
                    const int pos = pos0 + key, node = pos - prefix;
                    const bool there = plain || (pos < len && ((valid >> m) & 1));
                    if (!there) { a = make_float2(0.f, 0.f); v = a; }
                    a.y = fmaf(-8.f, a.x, a.y);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float &z = s[nb][m][2 * x + c];
                            z = fmaf(z, a.x * ra[nb][c], a.y * rb[nb][c]);
                            if (!plain && !(there && (node < 0 || ((s_seen[nb * 8 + 2 * t + c][node >> 5] >> (node & 31)) & 1u)))) z = -INFINITY;
                        }
                    vs[m][x] = v.x;
                    vm[m][x] = v.y;
                }
                const float l0 = att_level(vs[m][0]), l1 = att_level(vs[m][1]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float2 w0 = add2(make_float2(s[nb][m][0], s[nb][m][1]), make_float2(l0, l0));
                    const float2 w1 = add2(make_float2(s[nb][m][2], s[nb][m][3]), make_float2(l1, l1));
                    most[nb][0] = m ? max3(most[nb][0], w0.x, w1.x) : fmaxf(w0.x, w1.x);
                    most[nb][1] = m ? max3(most[nb][1], w0.y, w1.y) : fmaxf(w0.y, w1.y);
                }
            }
            bool move = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int c = 0; c < 2; ++c) move |= most[nb][c] > top[nb][c] + kNarrowSlack;
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float f[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float now = fmaxf(most[nb][c], top[nb][c]);
#pragma unroll
                        for (int q = 4; q < 32; q <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, q));
                        f[c] = ex2f(top[nb][c] - now);
                        top[nb][c] = now;
                        sum[nb][c] *= f[c];
                        mids[nb][c] *= f[c];
                        ones[nb][c] *= f[c];
                    }
#pragma unroll
                    for (int n = 0; n < MT; ++n) { o[nb][n][0] *= f[0]; o[nb][n][1] *= f[1]; o[nb][n][2] *= f[0]; o[nb][n][3] *= f[1]; }
                }
            }
            uint32_t pb[NB][2][2];                  // weights as operands: (row g, keys 2 t and 2 t + 1 of eight)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        float w[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float z = s[nb][m][2 * x + c];
                            const float p = ex2f(z - top[nb][c]);
                            sum[nb][c] += p;
                            // (the parameters of a key that is not seen may be anything)
                            if (plain || z != -INFINITY) mids[nb][c] = fmaf(p, vm[m][x], mids[nb][c]);
                            w[c] = plain || z != -INFINITY ? p * vs[m][x] : 0.f;
                        }
                        pb[nb][m][x] = transpose8(half2_bits(w[0], w[1]));
                    }
                }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    mma_f16(ones[nb], 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, pb[nb][m][0], pb[nb][m][1]);
                const unsigned char *codes = stage + kNarrowKeys * RB + 16 * m * RB;
                const int rows[4] = {ka, kb, 8 + ka, 8 + kb};
                uint32_t w[4][2];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (D == 128) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(codes + rows[q] * RB + swizzle(rows[q], g >> 1) * 16 + (g & 1) * 8);
                        w[q][0] = v.x; w[q][1] = v.y;
                    } else {
                        w[q][0] = w[q][1] = *reinterpret_cast<const uint32_t *>(codes + rows[q] * RB + g * 4);
                    }
                }
                // a tile's rows g and g + 8: with D = 128 code n of words 2 g and 2 g + 1, with D = 64 codes n and n + 4 of word g
#pragma unroll
                for (int hf = 0; hf < D / 64; ++hf) {
                    const int lo = hf ? 0x7632 : 0x5410, hi = D == 128 ? lo : 0x7632;
                    uint32_t x[4] = {__byte_perm(w[0][0], w[1][0], lo), __byte_perm(w[0][1], w[1][1], hi),
                                     __byte_perm(w[2][0], w[3][0], lo), __byte_perm(w[2][1], w[3][1], hi)};
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint32_t mask = n & 1 ? 0x00f000f0u : 0x000f000fu;
                        if (n == 2) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) x[q] >>= 8;
                        }
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
                            mma_f16(o[nb][4 * hf + n], x[0] & mask, x[1] & mask, x[2] & mask, x[3] & mask, pb[nb][m][0], pb[nb][m][1]);
                    }
                }
            }
        };

        int slot = 0, fill = STAGES - 1;
        for (int i = 0; i < n_chunks; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();                           // every lane's copies of chunk i are there, and chunk i - 1 is done with
            const unsigned char *stage = ring + slot * STAGE;
            const int valid = s_valid[warp][slot];
            issue(i + STAGES - 1, fill);
            const int pos0 = (k0 + i) * kAttUnit + warp * kNarrowKeys;
            if (valid == 3 && pos0 + kNarrowKeys <= prefix) chunk(std::true_type(), stage, pos0, valid);
            else chunk(std::false_type(), stage, pos0, valid);
            slot = slot == STAGES - 1 ? 0 : slot + 1;
            fill = fill == STAGES - 1 ? 0 : fill + 1;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
        // this warp's result as numbers, into its own ring
        float *s_out = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float l = sum[nb][c], z = mids[nb][c];
#pragma unroll
                for (int q = 4; q < 32; q <<= 1) {
                    l += __shfl_xor_sync(0xffffffffu, l, q);
                    z += __shfl_xor_sync(0xffffffffu, z, q);
                }
                const int row = nb * 8 + 2 * t + c;
                const float fixed = fmaf(-8.f, ones[nb][c], z);
                float *dst = s_out + row * D + g * (D / 8);
#pragma unroll
                for (int x = 0; x < 2; ++x)         // the tile's rows g, then its rows g + 8
#pragma unroll
                    for (int n = 0; n < MT; n += 4) {
                        float4 v;
                        v.x = fmaf(o[nb][n][2 * x + c], 16777216.f, fixed);
                        v.y = fmaf(o[nb][n + 1][2 * x + c], 1048576.f, fixed);
                        v.z = fmaf(o[nb][n + 2][2 * x + c], 16777216.f, fixed);
                        v.w = fmaf(o[nb][n + 3][2 * x + c], 1048576.f, fixed);
                        *reinterpret_cast<float4 *>(dst + x * MT + n) = v;
                    }
                if (g == 0) { s_top[warp][row] = top[nb][c]; s_sum[warp][row] = l; }
            }
        __syncthreads();
        // the four warps' results joined: D / 4 threads a row, four numbers each
        float *part = P.part + att_slot(k0) * part_floats(ROWS, D);
        for (int x = tid; x < ROWS * (D / 4); x += kNarrowWarps * 32) {
            const int r = x / (D / 4), c = (x % (D / 4)) * 4;
            if (row0 + r >= it.rows) break;
            float m = kNoTop;
#pragma unroll
            for (int w = 0; w < kNarrowWarps; ++w) m = fmaxf(m, s_top[w][r]);
            float l = 0.f;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kNarrowWarps; ++w) {
                const float f = att_factor(s_top[w][r], s_sum[w][r], m);
                const float4 v = *reinterpret_cast<const float4 *>(s_ring + w * STAGES * STAGE + (r * D + c) * 4);
                l = fmaf(f, s_sum[w][r], l);
                a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
            }
            if (it.whole) {
                att_store<DT, Rows>(P, it, row0 + r, c, a, m, l);
            } else {
                *reinterpret_cast<float4 *>(part + r * D + c) = a;
                if (c == 0) { part[ROWS * D + r] = m; part[ROWS * (D + 1) + r] = l; }
            }
        }
    }
}

// Joins the partial results of items that the cut divided: one CTA per item and eight of its rows, which
// finds the CTAs that worked on the item from the same arithmetic.
template <int DT, int D, int ROWS>
__global__ void __launch_bounds__(128)
join_kernel(const __grid_constant__ AttendParams P)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const uint32_t items = static_cast<uint32_t>(P.c.n_heads * P.n_blocks);
    const int b = static_cast<int>(blockIdx.x / items), item = static_cast<int>(blockIdx.x - b * items);
    const int len = att_len(P, b), units = att_units(len);
    const AttCut cut = att_cut(P, items, lane);
    const uint32_t u0 = att_before(P, cut.lead, b, lane) * items + static_cast<uint32_t>(item) * (units + cut.lead) + cut.lead;   // its first unit
    const int first = static_cast<int>(u0 / cut.per), last = static_cast<int>((u0 + units - 1) / cut.per);
    asm volatile("griddepcontrol.wait;" ::: "memory");   // (every thread: this kernel must not end before the one it follows)
    if (units == 0 || first == last) return;
    AttItem it = {};
    it.b = b;
    it.head = item / P.n_blocks;
    const int row0 = (item - it.head * P.n_blocks) * ROWS, r0 = blockIdx.y * 8;
    auto part_of = [&](int cta) { return P.part + static_cast<long long>(2 * cta + (cta == first ? 1 : 0)) * part_floats(ROWS, D); };
    for (int x = tid; x < 8 * (D / 4); x += 128) {
        const int r = r0 + x / (D / 4), c = (x % (D / 4)) * 4;
        if (row0 + r >= P.n_rows) break;
        float m = kNoTop;
        for (int k = first; k <= last; ++k) m = fmaxf(m, __ldcg(part_of(k) + ROWS * D + r));
        float l = 0.f;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = first; k <= last; ++k) {
            const float *part = part_of(k);
            const float lk = __ldcg(part + ROWS * (D + 1) + r);
            const float f = att_factor(__ldcg(part + ROWS * D + r), lk, m);
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + r * D + c));
            l = fmaf(f, lk, l);
            a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
        }
        att_store<DT, TreeRows>(P, it, row0 + r, c, a, m, l);
    }
}

}  // namespace mcsd
