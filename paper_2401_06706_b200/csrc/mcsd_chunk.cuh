// Attention of a chunk of new tokens over the paged 4-bit cache: the rows of a chunk as the narrow kernel sees them, the
// division of the work, and the joining of what it divided.
#pragma once

#include "mcsd_attend.cuh"

namespace mcsd {

struct ChunkParams {
    CacheParams c;
    const void *q;
    void *out;
    float *lse;                                     // of the attention: written (may be null); of the weights: read
    float *part;                                    // partial results, two slots per CTA
    struct ChunkJoin *joins;                        // per CTA: the block that it began and others end, if there is one
    float *weights;
    const int32_t *table, *start, *cu;
    long long ld_table, n_tokens;
    long long q_token, q_head, o_token, o_head;     // strides in elements
    int32_t batch, n_heads, max_pages, max_new;
    int32_t group;                                  // query heads per key/value head
    int32_t tokens;                                 // tokens of a block: as many as have all their rows in it
    int32_t least, most;                            // rows (tokens x group) that a sequence of this launch has
    int32_t n_ctas;                                 // CTAs the work is cut for
    int32_t lead;                                   // places of the cut a block costs beside its units
    int32_t last;                                   // tokens whose weights count, 0: all
    int32_t q_vec, o_vec;                           // rows of q may be read, those of out written in 16-byte vectors
    float scale, decay;
    float scale_part;                               // |scale| log2(e) = scale_part 2^scale_power, the part below 1
    int32_t scale_power;
    uint32_t wait_polls, test_extra;                // (as in AttendParams)
};

// A block that the cut divided: what the joining kernel needs to know, left by the CTA that has its first unit.
struct ChunkJoin { int b, head, row0, rows, last, pad[3]; };

// The new tokens of sequence b: the row of the first one, how many, the positions there are before them and with them.
struct ChunkSeq { int row, count, start, len; };
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkParams &P, int b)
{
    ChunkSeq s;
    const int first = __ldg(P.cu + b), next = __ldg(P.cu + b + 1);
    s.start = __ldg(P.start + b);
    const long long n = min(static_cast<long long>(next) - first, min(static_cast<long long>(P.max_new), P.n_tokens - first));
    s.row = first;
    s.count = s.start < 0 || first < 0 || n < 0 ? 0 : static_cast<int>(n);
    const long long there = static_cast<long long>(P.max_pages) << P.c.page_shift;
    s.len = static_cast<int>(min(static_cast<long long>(s.start) + s.count, there));
    return s;
}
// Positions that token i of the sequence sees.
__device__ __forceinline__ int chunk_sees(const ChunkSeq &s, int i) { return static_cast<int>(min(static_cast<long long>(s.start) + i + 1, static_cast<long long>(s.len))); }

// ---- the cut of the work
// An item is a block of `tokens` tokens of one (sequence, key/value head) with all rows of their heads; its units are the kAttUnit
// keys each that its last token sees.  Later blocks see more.  A place is a key: block j of a sequence has lead + start +
// (j + 1) tokens of them (the last one may have less to do), so that the places before a block are a polynomial of j and a CTA finds
// what it has without a table.  All blocks, one sequence after the other, are cut into runs of equal length, one per CTA; a unit
// belongs to the run that holds its first place.  The lengths are read on the device: a captured call follows them.
typedef unsigned long long ChunkPlace;
struct ChunkCut { ChunkPlace span, per; };
__device__ __forceinline__ int chunk_blocks(const ChunkParams &P, const ChunkSeq &s)
{
    const long long rows = static_cast<long long>(s.count) * P.group;
    return rows < P.least || rows > P.most ? 0 : (s.count + P.tokens - 1) / P.tokens;
}
// Places of a block beside (j + 1) tokens, and those before block j.
__device__ __forceinline__ ChunkPlace chunk_base(const ChunkParams &P, const ChunkSeq &s) { return static_cast<ChunkPlace>(min(s.start, s.len)) + P.lead; }
__device__ __forceinline__ ChunkPlace chunk_before(const ChunkParams &P, ChunkPlace base, int j)
{
    return static_cast<ChunkPlace>(j) * base + static_cast<ChunkPlace>(P.tokens) * (static_cast<ChunkPlace>(j) * (j + 1) / 2);
}
__device__ __forceinline__ ChunkPlace chunk_places(const ChunkParams &P, int b)     // of one key/value head
{
    const ChunkSeq s = chunk_seq(P, b);
    return chunk_before(P, chunk_base(P, s), chunk_blocks(P, s));
}
__device__ __forceinline__ ChunkCut chunk_cut(const ChunkParams &P, int lane)
{
    ChunkCut cut;
    cut.span = 0;
    for (int b = lane; b < P.batch; b += 32) cut.span += chunk_places(P, b);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) cut.span += __shfl_xor_sync(0xffffffffu, cut.span, o);
    cut.span *= static_cast<ChunkPlace>(P.c.n_heads);
    cut.per = (cut.span + P.n_ctas - 1) / P.n_ctas;
    if (cut.per < kAttUnit) cut.per = kAttUnit;     // (no run without a unit's worth)
    return cut;
}

// Where place `x` (below the span) lies: sequence, head, block, the place in the block, the block's places.
struct ChunkSpot { ChunkSeq s; int b, head, block; ChunkPlace at, places; };
__device__ __forceinline__ void chunk_block(const ChunkParams &P, ChunkSpot &t, ChunkPlace x)
{
    // the block: the root of tokens / 2 j^2 + (base + tokens / 2) j = x, put right where the rounding was wrong
    const ChunkPlace base = chunk_base(P, t.s);
    const double half = 0.5 * P.tokens, lin = static_cast<double>(base) + half;
    int j = static_cast<int>((sqrt(lin * lin + 4.0 * half * static_cast<double>(x)) - lin) / (2.0 * half));
    while (j > 0 && chunk_before(P, base, j) > x) --j;
    while (chunk_before(P, base, j + 1) <= x) ++j;
    t.block = j;
    t.at = x - chunk_before(P, base, j);
    t.places = base + static_cast<ChunkPlace>(j + 1) * P.tokens;
}
__device__ __forceinline__ ChunkSpot chunk_find(const ChunkParams &P, ChunkPlace x, int lane)
{
    ChunkSpot t;
    const ChunkPlace heads = static_cast<ChunkPlace>(P.c.n_heads);
    for (int b0 = 0;; b0 += 32) {
        const ChunkPlace n = b0 + lane < P.batch ? chunk_places(P, b0 + lane) * heads : 0;
        ChunkPlace incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const ChunkPlace up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        const unsigned past = __ballot_sync(0xffffffffu, incl > x);
        if (past || b0 + 32 >= P.batch) {
            const int who = past ? __ffs(past) - 1 : 31;
            t.b = b0 + who;
            x -= __shfl_sync(0xffffffffu, incl - n, who);
            const ChunkPlace one = __shfl_sync(0xffffffffu, n, who) / heads;
            t.head = static_cast<int>(x / one);
            t.s = chunk_seq(P, t.b);
            chunk_block(P, t, x - t.head * one);
            return t;
        }
        x -= __shfl_sync(0xffffffffu, incl, 31);
    }
}
// The next block after the one at `t`; false behind the last block of the sequence's last head.
__device__ __forceinline__ bool chunk_next(const ChunkParams &P, ChunkSpot &t)
{
    t.at = 0;
    if (++t.block >= chunk_blocks(P, t.s)) {
        t.block = 0;
        if (++t.head >= P.c.n_heads) return false;
    }
    t.places = chunk_base(P, t.s) + static_cast<ChunkPlace>(t.block + 1) * P.tokens;
    return true;
}
// Positions that the last token of the block sees, and the units they make (one for an empty block, whose rows are written too).
__device__ __forceinline__ int chunk_len(const ChunkParams &P, const ChunkSpot &t) { return chunk_sees(t.s, min((t.block + 1) * P.tokens, t.s.count) - 1); }
__device__ __forceinline__ int chunk_units(int len) { return max((len + kAttUnit - 1) / kAttUnit, 1); }
// Units whose first place is below place `at` of a block.
__device__ __forceinline__ int chunk_units_below(const ChunkParams &P, ChunkPlace at, int units)
{
    if (at <= static_cast<ChunkPlace>(P.lead)) return 0;
    const ChunkPlace k = (at - P.lead + kAttUnit - 1) / kAttUnit;
    return k < static_cast<ChunkPlace>(units) ? static_cast<int>(k) : units;
}

// Key codes as halves, the eight of a word. Bits of a code in the mantissa of a subnormal number are a number without further ado; which bits
// matters: the matrix instructions align products, it seems, by the operands' exponents, and a subnormal number has that of 2^-14. One AND for
// two codes gives c 2^-24 and 16 c 2^-24, and an error of 4.5e-6 of gathered weights with fp16 queries (eleven bits each, windows of 32 tokens). At
// the top of the mantissa, c 2^-18, it is 3.6e-7, half as large as before with bf16 ones, and the shifts cost nothing that shows (weights of 32
// sequences of one token 25 us either way).
constexpr int kKeyExp = 18;
constexpr float kKeyUnit = 3.814697265625e-6f;      // 2^-18
__device__ __forceinline__ uint4 key_codes(uint32_t w)
{
    return make_uint4(w << 6 & 0x03c003c0u, w << 2 & 0x03c003c0u, w >> 2 & 0x03c003c0u, w >> 6 & 0x03c003c0u);
}

// Left by one thread of a CTA when it begins (nothing to join), and when it has begun a block that others end.
__device__ __forceinline__ void chunk_join_none(const ChunkParams &P) { P.joins[blockIdx.x].last = -1; }
__device__ __forceinline__ void chunk_join_note(const ChunkParams &P, const AttItem &it)
{
    if (it.whole || it.k0 > 0) return;
    ChunkJoin *j = P.joins + blockIdx.x;
    j->b = it.b; j->head = it.head; j->row0 = it.row0; j->rows = it.rows; j->last = it.last;
}

// The rows of a chunk, as the narrow kernel and its like see them: the mathematics are the narrow kernel's, a block's rows are tokens x query heads
// (8, 16 or 24 of them), and the part that differs by row is behind the block's first token. A sequence of one token with four heads to a
// key head reads its codes once: 64 sequences of 2 tokens over 4000 rows each, 8 key heads of 128, 80 us, 3.5 of the 6.55 TB/s that a copy has, 6 tokens 156; with
// lengths drawn from 1 to 4000 53 (2.9 TB/s) and 114.
struct ChunkRows {
    typedef ChunkParams Params;
    struct Walk {
        ChunkSpot t;
        ChunkPlace at, left, per;                   // place the walk has come to, places left of the run, places of a run
        bool fresh;
        __device__ __forceinline__ bool begin(const ChunkParams &P, int lane)
        {
            const ChunkCut cut = chunk_cut(P, lane);
            const ChunkPlace x = blockIdx.x * cut.per;
            if (x >= cut.span) return false;
            at = x;
            left = cut.span - x < cut.per ? cut.span - x : cut.per;
            per = cut.per;
            t = chunk_find(P, x, lane);
            fresh = true;
            return true;
        }
        template <int ROWS>
        __device__ __forceinline__ bool next(const ChunkParams &P, int lane, AttItem &it)
        {
            for (;;) {
                if (!fresh) {                       // to the block after the one before
                    const ChunkPlace had = t.places - t.at;
                    if (left <= had) return false;
                    left -= had;
                    at += had;
                    if (!chunk_next(P, t)) {
                        int b = t.b + 1;
                        while (b < P.batch && chunk_places(P, b) == 0) ++b;
                        if (b >= P.batch) return false;         // (cannot be: there are places left)
                        t.b = b;
                        t.s = chunk_seq(P, b);
                        t.head = t.block = 0;
                        t.places = chunk_base(P, t.s) + P.tokens;
                    }
                }
                fresh = false;
                const ChunkPlace to = t.at + (left < t.places - t.at ? left : t.places - t.at);
                const int len = chunk_len(P, t), units = chunk_units(len);
                it.k0 = chunk_units_below(P, t.at, units);
                it.k1 = chunk_units_below(P, to, units);
                if (it.k0 >= it.k1) continue;
                it.b = t.b;
                it.head = t.head;
                it.len = len;
                it.row0 = t.block * P.tokens * P.group;
                it.rows = min((t.block + 1) * P.tokens, t.s.count) * P.group;
                it.tail = chunk_sees(t.s, t.block * P.tokens);
                it.whole = it.k0 == 0 && it.k1 == units;
                it.last = static_cast<int>((at - t.at + P.lead + static_cast<ChunkPlace>(units - 1) * kAttUnit) / per);
                return true;
            }
        }
        template <int ROWS>
        __device__ __forceinline__ bool here(const ChunkParams &P, int lane, AttItem &it) { return next<ROWS>(P, lane, it); }
        __device__ __forceinline__ void on(const ChunkParams &, int) {}
    };
    static __device__ __forceinline__ void begun(const ChunkParams &P) { chunk_join_none(P); }
    static __device__ __forceinline__ void divided(const ChunkParams &P, const AttItem &it) { chunk_join_note(P, it); }
    static __device__ __forceinline__ long long q_at(const ChunkParams &P, const AttItem &it, int row)
    {
        const int i = row / P.group, h = it.head * P.group + (row - i * P.group);
        return (static_cast<long long>(__ldg(P.cu + it.b)) + i) * P.q_token + h * P.q_head;
    }
    // Positions behind `tail` that a row sees: those up to its own (the first token of the block is at tail - 1, where it is there).
    static __device__ __forceinline__ void see(const ChunkParams &P, const AttItem &it, int row, uint32_t *seen)
    {
        const int n = row < it.rows ? row / P.group - it.row0 / P.group : 0;         // (fewer than 32)
        seen[0] = (1u << n) - 1u;
    }
    static __device__ __forceinline__ long long out_at(const ChunkParams &P, const AttItem &it, int row)
    {
        const int i = row / P.group, h = it.head * P.group + (row - i * P.group);
        return (static_cast<long long>(__ldg(P.cu + it.b)) + i) * P.o_token + h * P.o_head;
    }
    static __device__ __forceinline__ long long lse_at(const ChunkParams &P, const AttItem &it, int row)
    {
        const int i = row / P.group;
        return (static_cast<long long>(__ldg(P.cu + it.b)) + i) * P.n_heads + it.head * P.group + (row - i * P.group);
    }
};

// Joins the partial results of blocks that the cut divided: a CTA for eight (D = 128) or sixteen rows of each. Which blocks those are, the kernel
// before notes in the workspace (looking for them again, with dependent loads of lengths, took 62 -> 79 us of 64 tokens over 4000 rows of 4 sequences). The
// parts of a block lie one after the other by CTA and are added up in that order. Bound by latency: 3 to 4 us, most of them behind the end of that kernel.
constexpr int kChunkJoinThreads = 256;
template <int DT, int D, int ROWS>
__global__ void __launch_bounds__(kChunkJoinThreads)
chunk_join_kernel(const __grid_constant__ ChunkParams P)
{
    constexpr int TPR = D / 4;                      // threads of a row, four numbers each
    const int first = blockIdx.x, r = blockIdx.y * (kChunkJoinThreads / TPR) + threadIdx.x / TPR, c = (threadIdx.x % TPR) * 4;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // (every thread: this kernel must not end before the one it follows)
    const ChunkJoin j = P.joins[first];
    if (j.last < 0 || r >= min(ROWS, j.rows - j.row0)) return;
    AttItem it = {};
    it.b = j.b; it.head = j.head; it.rows = j.rows;
    auto part_of = [&](int cta) { return P.part + static_cast<long long>(2 * cta + (cta == first ? 1 : 0)) * part_floats(ROWS, D); };
    // (relative to the largest reference so far: one pass over the parts)
    float m = kNoTop, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int k = first; k <= j.last; ++k) {
        const float *part = part_of(k);
        const float mk = __ldcg(part + ROWS * D + r), lk = __ldcg(part + ROWS * (D + 1) + r);
        const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + r * D + c));
        const float top = fmaxf(m, mk), f = att_factor(m, l, top), g = att_factor(mk, lk, top);
        m = top;
        l = fmaf(f, l, g * lk);
        a.x = fmaf(f, a.x, g * v.x); a.y = fmaf(f, a.y, g * v.y); a.z = fmaf(f, a.z, g * v.z); a.w = fmaf(f, a.w, g * v.w);
    }
    att_store<DT, ChunkRows>(P, it, j.row0 + r, c, a, m, l);
}

}  // namespace mcsd
