// Tree attention for many rows per key/value head: 128 rows a block on the tcgen05 tensor cores.
#pragma once

#include "mcsd_attend.cuh"

namespace mcsd {

// (the compiler leaves the larger of these lambdas as calls otherwise)
#define MCSD_INLINE __attribute__((always_inline))

constexpr int kWideRows = 128;
constexpr int kWideThreads = 640;                   // 8 softmax warps, 8 decoding warps, 2 that issue (and 2 beside them)
constexpr int kWideStages = 2;                      // decoded units
constexpr int kWideAhead = 4;                       // units whose codes are on their way to shared memory
constexpr float kWideSpread = 4.f;                  // octaves of value scales that one number may stand for
template <int D> constexpr int kWideTile = kAttUnit * D * 2;                       // bytes of a decoded tile of keys or values
template <int D> constexpr int kWideSmem = 1024 + kWideStages * (2 * kWideTile<D> + kAttUnit * 16) + kWideAhead * kAttUnit * (D + 8) + kWideRows * (MCSD_MAX_NODES / 32) * 4;

// ---- tensor memory and tcgen05
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Products are issued by a whole warp, converged, with one thread elected for each instruction (always the same
// one): what describes them then stays in uniform registers, which a single-threaded loop has to
// refill for every instruction (it measured 390 against 339 us on 181 x 4 rows over 16001 positions).
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// D (tensor memory) (+)= A (tensor memory, 128 rows x 16) * B (shared memory, described by two words), halves in, float32 out.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint32_t b_low, uint32_t b_high, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 b;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b_low), "r"(b_high), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
#define MCSD_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define MCSD_W8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// Columns of this warp's 32 lanes, lane i of the warp row i.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"   // (in the same statement: the registers hold nothing before it)
                 : MCSD_R8(v, 0), MCSD_R8(v, 8), MCSD_R8(v, 16), MCSD_R8(v, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t at, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
                 "tcgen05.wait::ld.sync.aligned;" : MCSD_R8(v, 0) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&v)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::MCSD_W8(v, 0), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"   // (in the same statement: the registers hold nothing before it)
                 : MCSD_R8(v, 0), MCSD_R8(v, 8) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::MCSD_W8(v, 0), MCSD_W8(v, 8), "r"(at) : "memory");
}
#undef MCSD_R8
#undef MCSD_W8

// Descriptor of an operand in shared memory in rows of 128 bytes whose 16-byte chunks are exchanged by the
// row's index mod 8 (1024-byte groups of eight rows): the low word (advanced by bytes / 16) and the high one. `lead` is the
// distance to the next 64 numbers of the contiguous side where that side is not the summed one.
__device__ __forceinline__ uint32_t tc_operand(uint32_t at, uint32_t lead) { return ((at & 0x3ffffu) >> 4) | (lead >> 4) << 16; }
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
// 128 x n, half operands, float32 result; `outer`: B's contiguous side is n, not the summed one.
__host__ __device__ constexpr uint32_t tc_shape(int n, bool outer) {
    return 1u << 4 | (outer ? 1u << 16 : 0u) | static_cast<uint32_t>(n >> 3) << 17 | static_cast<uint32_t>(kWideRows >> 4) << 24;
}

// Registers per thread of the groups of four warps: the kernel is launched with 96 each, the groups that decode and issue
// give away what the softmax groups take (2 x 168 + 2 x 56 + 32 = 5 x 96).
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Bounded wait of a warp of the roles below (every poll may suspend it for a microsecond, so the bound is a few
// seconds unless a test shortens it).  Once one has given up every wait returns at once: the roles run to their end, whatever they compute, nobody
// is left waiting, and the rows are written as NaN.
__device__ __forceinline__ void wide_wait(uint32_t bar, uint32_t parity, volatile int *dead, uint32_t polls) {
    for (uint32_t i = 0; i < polls; ++i) {
        if (mbar_try_wait(bar, parity)) break;
        if ((i & 31) == 31 && *dead) break;
        if (i == polls - 1) *dead = 1;
    }
    __syncwarp();
}
// One arrival for the whole warp, behind what all its lanes did.
__device__ __forceinline__ void warp_arrive(uint32_t bar, int lane) {
    __syncwarp();
    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// One CTA per SM, work cut as for the narrow kernel, in units of 128 keys. Roles:
//   decoding warps  (four for keys, four for values, 32 rows of every unit each) copy codes to rings of their own, four units
//                   ahead, and turn them into operands in shared memory: a 4-bit code becomes a subnormal half by one AND (see
//                   the narrow kernel), those of the values less 8, an exact subtraction; codes stay in the order the
//                   ANDs give them, which Q and the output undo;
//   issuing warps   one per softmax group: S = Q K^T and O += P V by tcgen05.mma, Q and P from tensor memory, K and V
//                   from shared memory; the scores of a unit as soon as those of the unit before are read;
//   softmax groups  A and B (128 threads each, one row per thread) take keys 0..63 and 64..127 of every unit, each with
//                   maxima, sums and an O of its own, so that neither waits for the other: while one exponentiates, the
//                   tensor cores work for the other. A joins both at the end of an item.
// Scale and mid of a key enter the scores in float32; the weight p vscale is rounded to half once. The
// reference of a row's exponents follows its largest weight over the keys that it sees, as in the narrow kernel, and moves only when
// it is exceeded by 2^kNarrowSlack. Where a row sees all keys of a unit and their value scales lie within 2^kWideSpread of each
// other, the largest score plus the largest scale's log2 stands for that weight (one addition; 2^kWideSpread above it at most, which
// half's range has room for); elsewhere it is formed key by key.
// Tensor memory (columns; all 512 are taken, so that the first is column 0): S of A, S of B (64 each), O of A, O of B (D
// each), P of A, P of B (32 each), Q (D / 2).
// Measured on 724 rows x 8 key heads x 4 sequences of up to 16001 positions: 283 us, 482 TFLOP/s, 0.29 of the measured
// peak. The products take about a fifth of the time; what bounds it is the chain of a softmax group for a unit (scores
// read, exponentials, weights written: some 2000 cycles of two warps per scheduler) and the hand-overs around
// it. With the work cut by units alone it took 297 us, without the copies four units ahead 345 us, with products issued by a
// single thread 390 us. Left out: sixteen
// softmax warps of sixteen rows in fragment layout (a quarter of the parameter loads, 322 us; 20 % slower than this
// form on prefixes of 2000, where the tree's own units weigh more), separate rings for keys and values (328 us). The softmax warps spill
// 36 bytes a thread.
template <int DT, int D>
__global__ void __launch_bounds__(kWideThreads, 1)
wide_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int TILE = kWideTile<D>, RB = D / 2;
    constexpr uint32_t kS = 0, kO = 128, kP = 128 + 2 * D, kQ = 192 + 2 * D, kColumns = 512;
    extern __shared__ unsigned char s_raw[];
    __shared__ __align__(8) unsigned long long s_bar[2 * kWideStages + 12];
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    __shared__ uint32_t s_valid[kWideStages][4];    // keys of a stage that are there
    __shared__ float2 s_level[kWideStages][4];      // log2 of the largest and of the smallest value scale of 32 keys
    __shared__ float4 s_other[kWideRows];           // reference and sums of group B at the end of an item
    __shared__ float2 s_row[kWideRows];             // of a row: log2 units per unit, and sum of q in accumulator units
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    unsigned char *base = s_raw + ((1024 - (smem_u32(s_raw) & 1023)) & 1023);
    unsigned char *s_tiles = base;                                              // [stages][keys, values]
    float4 *s_param = reinterpret_cast<float4 *>(base + 2 * kWideStages * TILE);  // [stages][64 pairs of keys]{key, value}
    uint32_t(*s_seen)[MCSD_MAX_NODES / 32] = reinterpret_cast<uint32_t(*)[MCSD_MAX_NODES / 32]>(
        base + 2 * kWideStages * TILE + kWideStages * kAttUnit * 16);
    unsigned char *s_codes = reinterpret_cast<unsigned char *>(s_seen + kWideRows);   // [decoding warps][kWideAhead]{codes, parameters}

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = smem_u32(s_bar);
    const uint32_t b_full = bars, b_empty = b_full + 8 * kWideStages, b_s = b_empty + 8 * kWideStages, b_read = b_s + 16, b_p = b_s + 32,
                   b_o = b_s + 48, b_ready = b_s + 64, b_free = b_s + 72, b_merge = b_s + 80, b_end = b_s + 88;
    if (tid == 0) {
        for (int i = 0; i < kWideStages; ++i) {
            mbar_init(b_full + 8 * i, 8);           // (arrivals of warps)
            mbar_init(b_empty + 8 * i, 10);         // the products of both groups, and the softmax warps, which read the parameters
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_read + 8 * i, 4);
            mbar_init(b_p + 8 * i, 4);
            mbar_init(b_o + 8 * i, 1);
        }
        mbar_init(b_ready, 4 + P.test_extra);       // (0 but in a test of the expiry path: arrivals that never come)
        mbar_init(b_free, 4);
        mbar_init(b_merge, 4);
        mbar_init(b_end, 2);
        fence_mbar_init();
        s_dead = 0;
    }
    if (warp == 16) tmem_alloc(smem_u32(&s_tmem), kColumns);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    constexpr uint32_t tmem = 0;
    volatile int *dead = &s_dead;
    if (s_tmem != tmem) *dead = 1;                  // (cannot be: all columns are this CTA's)

    const int ps = 1 << P.c.page_shift;
    const uint32_t items = static_cast<uint32_t>(P.c.n_heads * P.n_blocks);
    const AttCut cut = att_cut(P, items, lane);
    const bool any = cut.span != 0 && blockIdx.x <= (cut.span - 1) / cut.per;     // (runs before the last one are whole)
    const uint32_t u_begin = any ? blockIdx.x * cut.per : 0, u_end = any ? (cut.span - u_begin < cut.per ? cut.span : u_begin + cut.per) : 0;

    // Every role goes over the same items; f(sequence, length, head, first row, first unit, last unit + 1, whole item).
    auto for_items = [&](auto f) {
        if (u_begin >= u_end) return;
        AttCursor cur = att_find(P, cut, u_begin, items, lane);
        for (uint32_t u = u_begin; u < u_end;) {
            const AttPiece piece = att_piece(cut, cur, u_end - u);
            if (piece.k1 <= 0) break;
            const int head = piece.item / P.n_blocks;
            f(cur.b, cur.len, head, (piece.item - head * P.n_blocks) * kWideRows, piece.k0, piece.k1, piece.k0 == 0 && piece.k1 == piece.units);
            u += piece.places;
            cur.at += piece.places;
            if (u < u_end && cur.at >= cur.places * items) cur = att_find(P, cut, u, items, lane);
        }
    };

    if (warp >= 8 && warp < 16) {
        // ------------------------------------------------------------ decoding
        regs_down<56>();
        // A warp has 32 keys of every unit, key or value rows: lane by lane, 16 bytes of codes at 16 (lane + 32 i) of
        // the rows of sixteen keys, so that a load is contiguous, and the parameters of key `lane`.
        constexpr int CH = RB / 16;                 // 16-byte chunks of a row: 2 or 4
        const int which = (warp >> 2) & 1, key0 = (warp & 3) * 32;       // which: 0 key rows, 1 value rows
        const int c = lane % CH;
        int stage = 0;
        uint32_t phase = 1;                         // (the first round of stages is free)
        for_items([&](int b, int len, int head, int, int k0, int k1, bool) MCSD_INLINE {
            const int32_t *table = P.table + b * P.ld_table;
            const unsigned char *pool = P.c.pages + static_cast<long long>(head) * kv_block_bytes(D, ps);
            // page of this lane's half (lanes 0..15: the first sixteen keys)
            auto page_of = [&](int k) MCSD_INLINE {
                const int pos = k * kAttUnit + key0 + (lane & 16);
                return k < k1 && pos < len ? __ldg(table + (pos >> P.c.page_shift)) : -1;
            };
            // Rows of unit k are copied to this warp's own ring, kWideAhead units ahead; a lane reads back what it copied itself.
            unsigned char *ring = s_codes + (warp & 7) * kWideAhead * 32 * (RB + 4);
            uint32_t there = 0u;                    // bit `slot`: this lane's key of that unit is in the cache
            int k = k0, page = -1;                  // page: of the unit asked for next
            auto issue = [&](int unit, int slot) MCSD_INLINE {
                const int pos = unit * kAttUnit + key0 + lane;
                unsigned char *to = ring + slot * 32 * (RB + 4);
                if (unit < k1) {
                    const bool ok = static_cast<unsigned>(page) < static_cast<unsigned>(P.c.n_pages) && pos < len;
                    there = (there & ~(1u << slot)) | static_cast<uint32_t>(ok) << slot;
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int p = __shfl_sync(0xffffffffu, page, 16 * hf);
                        if (static_cast<unsigned>(p) < static_cast<unsigned>(P.c.n_pages)) {
                            const unsigned char *src = pool + p * P.c.page_stride + (which * ps + ((unit * kAttUnit + key0 + 16 * hf) & (ps - 1))) * RB + lane * 16;
#pragma unroll
                            for (int i = 0; i < CH / 2; ++i) cp_async16(smem_u32(to + (hf * (CH / 2) + i) * 512 + lane * 16), src + 512 * i);
                        }
                    }
                    if (ok) cp_async4(to + 32 * RB + lane * 4, pool + page * P.c.page_stride + ps * D + (which * ps + (pos & (ps - 1))) * 4);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            int pages[kWideAhead + 1];
#pragma unroll
            for (int i = 0; i <= kWideAhead; ++i) pages[i] = page_of(k + i);
#pragma unroll
            for (int i = 0; i < kWideAhead; ++i) {
                page = pages[i];
                issue(k + i, i);
            }
            page = pages[kWideAhead];
            int slot = 0;
            for (; k < k1; ++k) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kWideAhead - 1) : "memory");
                const unsigned char *from = ring + slot * 32 * (RB + 4);
                wide_wait(b_empty + 8 * stage, phase, dead, P.wait_polls);
#pragma unroll
                for (int i = 0; i < CH; ++i) {      // 16 bytes of codes are four 16-byte chunks of operands
                    const int key = key0 + (i / (CH / 2)) * 16 + (i % (CH / 2)) * (32 / CH) + lane / CH;
                    unsigned char *tile = s_tiles + (2 * stage + which) * TILE + key * 128;
                    // (with four chunks a row, lanes 2 and 3 take their words in another order: no two lanes of eight meet in a bank)
                    const bool turn = CH == 4 && (c & 2);
                    const uint4 v = *reinterpret_cast<const uint4 *>(from + i * 512 + lane * 16);
                    const uint32_t w[4] = {turn ? v.z : v.x, turn ? v.w : v.y, turn ? v.x : v.z, turn ? v.y : v.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t y = w[j] >> 8;
                        uint32_t h[4] = {w[j] & 0x000f000fu, w[j] & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u};
                        if (which) {                // less 8 (in units of 2^-24, the odd ones of 2^-20): exact
                            const uint32_t eight[2] = {0x00080008u, 0x00800080u};
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&h[q]), *reinterpret_cast<const __half2 *>(&eight[q & 1]));
                                h[q] = *reinterpret_cast<const uint32_t *>(&d);
                            }
                        }
                        const int chunk = 4 * c + (turn ? j ^ 2 : j);
                        *reinterpret_cast<uint4 *>(tile + (chunk >> 3) * (kAttUnit * 128) + (((chunk & 7) ^ (key & 7)) << 4)) =
                            make_uint4(h[0], h[1], h[2], h[3]);
                    }
                }
                // scale and mid - 8 scale of the key, scale and mid of the value, in pairs of keys
                const bool mine = (there >> slot) & 1u;
                const float2 p = mine ? __half22float2(*reinterpret_cast<const __half2 *>(from + 32 * RB + lane * 4)) : make_float2(0.f, 0.f);
                const int key = key0 + lane;
                float *par = reinterpret_cast<float *>(s_param + stage * kAttUnit + (key >> 1) * 2 + which) + (key & 1);
                par[0] = p.x;
                par[2] = which ? p.y : fmaf(-8.f, p.x, p.y);
                if (which == 0) {
                    const uint32_t keys = __ballot_sync(0xffffffffu, mine);
                    if (lane == 0) s_valid[stage][warp & 3] = keys;
                } else {
                    const float level = att_level(p.x);
                    const float2 ends = make_float2(warp_max(level), -warp_max(-level));
                    if (lane == 0) s_level[stage][warp & 3] = ends;
                }
                fence_proxy_async();
                warp_arrive(b_full + 8 * stage, lane);
                if (++stage == kWideStages) { stage = 0; phase ^= 1; }
                issue(k + kWideAhead, slot);        // (what this lane had there is read)
                page = page_of(k + kWideAhead + 1); // (in flight until the next unit is asked for)
                slot = slot == kWideAhead - 1 ? 0 : slot + 1;
            }
        });
    } else if (warp >= 16) {
        // ------------------------------------------------------------ issuing
        regs_down<32>();
        const int x = warp - 16;                    // the group it issues for
        if (x < 2) {
            int stage = 0;
            uint32_t phase = 0, n = 0, it = 0;      // n: units so far
            auto scores = [&](int stage, uint32_t phase) {
                wide_wait(b_full + 8 * stage, phase, dead, P.wait_polls);
                tc_after_sync();
                const uint32_t at = tc_operand(smem_u32(s_tiles) + stage * 2 * TILE + x * 64 * 128, 16);
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    tc_mma(tmem + kS + 64 * x, tmem + kQ + 8 * s, at + (s >> 2) * (kAttUnit * 128 / 16) + (s & 3) * 2, kOperandHigh, tc_shape(64, false), s > 0);
                tc_commit(b_s + 8 * x);
            };
            for_items([&](int, int, int, int, int k0, int k1, bool) {
                wide_wait(b_ready, it & 1, dead, P.wait_polls);
                scores(stage, phase);
                for (int k = k0; k < k1; ++k, ++n) {
                    const int here = stage;
                    if (++stage == kWideStages) { stage = 0; phase ^= 1; }
                    if (k + 1 < k1) {               // the group has read the scores of this unit: those of the next
                        wide_wait(b_read + 8 * x, n & 1, dead, P.wait_polls);
                        scores(stage, phase);
                    }
                    wide_wait(b_p + 8 * x, n & 1, dead, P.wait_polls);          // its weights are written
                    tc_after_sync();
                    const uint32_t at = tc_operand(smem_u32(s_tiles) + (here * 2 + 1) * TILE + x * 64 * 128, kAttUnit * 128);
#pragma unroll
                    for (int s = 0; s < 4; ++s)
                        tc_mma(tmem + kO + D * x, tmem + kP + 32 * x + 8 * s, at + s * (16 * 128 / 16), kOperandHigh, tc_shape(D, true), k > k0 || s > 0);
                    tc_commit(b_o + 8 * x);
                    tc_commit(b_empty + 8 * here);
                }
                ++it;
            });
            // What was issued, by both warps, ends before its memory is given back. (Where no wait expires, the softmax groups have
            // waited for the products already; where one does, it may be the last of all, after this warp is through.)
            tc_commit(b_end);
            for (uint32_t i = 0; i < kWaitPolls && !__all_sync(0xffffffffu, mbar_try_wait(b_end, 0)); ++i) {}
        }
    } else {
        // ------------------------------------------------------------ softmax
        regs_up<168>();
        const int x = warp >> 2;                    // 0: group A, 1: group B
        const int r = tid & 127;                    // row of the block = lane of tensor memory
        const uint32_t mine = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + mine + kS + 64 * x, t_o = tmem + mine + kO + D * x, t_p = tmem + mine + kP + 32 * x;
        int stage = 0;
        uint32_t phase = 0, n = 0, it = 0;
        for_items([&](int b, int len, int head, int row0, int k0, int k1, bool whole) {
            const int row = row0 + r;
            const bool busy = row0 + (r & ~31) < P.n_rows;        // this warp has rows
            const int prefix = P.prefix_len[b];
            const int node = row < P.n_rows ? row / P.group : 0, h = head * P.group + (row - node * P.group);
            float rho, ra;                          // score in log2 units: ra (scale acc + (mid - 8 scale) rho)
            if (x == 0) {
                // Q to tensor memory, scaled by a power of two to the top of half's range (and to a positive softmax scale)
                uint4 raw[D / 8];
#pragma unroll
                for (int c = 0; c < D / 8; ++c) raw[c] = make_uint4(0u, 0u, 0u, 0u);
                if (row < P.n_rows) {
                    const long long at = b * P.q_seq + node * P.q_node + h * P.q_head;
                    if (P.q_vec) {
#pragma unroll
                        for (int c = 0; c < D / 8; ++c) raw[c] = (reinterpret_cast<const uint4 *>(static_cast<const char *>(P.q) + 2 * at))[c];   // (not the read-only path: out may be q)
                    } else {
                        const unsigned short *src = static_cast<const unsigned short *>(P.q) + at;
#pragma unroll
                        for (int c = 0; c < D / 8; ++c)
                            raw[c] = make_uint4(src[8 * c] | src[8 * c + 1] << 16, src[8 * c + 2] | src[8 * c + 3] << 16,
                                                src[8 * c + 4] | src[8 * c + 5] << 16, src[8 * c + 6] | src[8 * c + 7] << 16);
                    }
                }
                for (int i = 0; i * 32 < P.n_nodes; ++i) s_seen[r][i] = 0u;
                for (int a = row < P.n_rows ? node : -1; a >= 0; a = P.parent[a]) s_seen[r][a >> 5] |= 1u << (a & 31);
                float most = 0.f, sum = 0.f;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    float v[8];
                    Elem<DT>::unpack(raw[c], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) { most = fmaxf(most, fabsf(v[i])); sum += v[i]; }
                }
                int e = most > 0.f ? static_cast<int>(__float_as_uint(most) >> 23) - 126 : 0;
                e = max(min(e, 112), -110);
                const float up = __int_as_float((127 + 15 - e) << 23) * (P.scale < 0.f ? -1.f : 1.f);
                ra = ldexpf(fabsf(P.scale) * 1.4426950408889634f, e - 15 + 24);
                rho = sum * up * 5.9604644775390625e-8f;          // 2^-24
#pragma unroll
                for (int c0 = 0; c0 < D / 32; ++c0) {
                    uint32_t out[16];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {                 // eight numbers, one word of codes
                        float v[8];
                        Elem<DT>::unpack(raw[4 * c0 + c], v);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float f = i & 1 ? up * 0.0625f : up;
                            out[4 * c + i] = half2_bits(v[i] * f, v[i + 4] * f);
                        }
                    }
                    __syncwarp();
                    tmem_store16(tmem + mine + kQ + 16 * c0, out);
                }
                s_row[r] = make_float2(ra, rho);
                __syncwarp();
                tc_wait_st();
                tc_before_sync();
                warp_arrive(b_ready, lane);
            } else {
                wide_wait(b_ready, it & 1, dead, P.wait_polls);
                ra = s_row[r].x;
                rho = s_row[r].y;
            }
            float ref = kNoTop, sum = 0.f, mids = 0.f;
            for (int k = k0; k < k1; ++k, ++n) {
                wide_wait(b_s + 8 * x, n & 1, dead, P.wait_polls);
                wide_wait(b_full + 8 * stage, phase, dead, P.wait_polls);
                tc_after_sync();
                const float4 *par = s_param + stage * kAttUnit + 64 * x;       // two per pair of keys
                const int pos0 = k * kAttUnit + 64 * x;
                // see: keys this row sees; top: log2 of the largest value scale, where `plain`
                auto unit = [&](auto plain_tag, uint32_t see0, uint32_t see1, float top) {
                    constexpr bool plain = decltype(plain_tag)::value;
                    float2 y[32];
                    float most = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t acc[32];
                        tmem_load32(t_s + 32 * c, acc);
                        if (c == 1) {
                            tc_before_sync();
                            warp_arrive(b_read + 8 * x, lane);
                        }
                        const uint32_t see = c ? see1 : see0;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float4 kp = par[2 * (16 * c + j)];
                            const float2 off = __fmul2_rn(make_float2(kp.z, kp.w), make_float2(rho, rho));
                            float2 z = fma2(make_float2(__uint_as_float(acc[2 * j]), __uint_as_float(acc[2 * j + 1])), make_float2(kp.x, kp.y), off);
                            if (plain) {
                                most = max3(most, z.x, z.y);
                            } else {
                                const float4 vp = par[2 * (16 * c + j) + 1];
                                const float2 w = fma2(z, make_float2(ra, ra), make_float2(att_level(vp.x), att_level(vp.y)));
                                if ((see >> (2 * j)) & 1u) most = fmaxf(most, w.x);
                                if ((see >> (2 * j + 1)) & 1u) most = fmaxf(most, w.y);
                            }
                            y[16 * c + j] = z;
                        }
                    }
                    // O and P belong to this group once the product of the unit before is done
                    if (n > 0) wide_wait(b_o + 8 * x, (n - 1) & 1, dead, P.wait_polls);
                    tc_after_sync();
                    const float high = plain ? fmaf(most, ra, top) : most;
                    if (__any_sync(0xffffffffu, high > ref + kNarrowSlack)) {
                        const float now = fmaxf(ref, high);
                        const float f = ex2f(ref - now);
                        ref = now;
                        sum *= f;
                        mids *= f;
                        if (k > k0) {
#pragma unroll 1
                            for (int c = 0; c < D / 8; ++c) {     // (eight columns at a time: y holds most registers)
                                uint32_t o[8];
                                __syncwarp();
                                tmem_load8(t_o + 8 * c, o);
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_store8(t_o + 8 * c, o);
                            }
                        }
                    }
                    float2 s2 = make_float2(0.f, 0.f), m2 = make_float2(0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t w[16];
                        const uint32_t see = c ? see1 : see0;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float2 e = fma2(y[16 * c + j], make_float2(ra, ra), make_float2(-ref, -ref));
                            float2 p = make_float2(ex2f(e.x), ex2f(e.y));
                            float4 vp = par[2 * (16 * c + j) + 1];
                            if (!plain) {           // (the parameters of a key that is not seen may be anything)
                                if (!((see >> (2 * j)) & 1u)) { p.x = 0.f; vp.x = vp.z = 0.f; }
                                if (!((see >> (2 * j + 1)) & 1u)) { p.y = 0.f; vp.y = vp.w = 0.f; }
                            }
                            s2 = add2(s2, p);
                            m2 = fma2(p, make_float2(vp.z, vp.w), m2);
                            const float2 q = __fmul2_rn(p, make_float2(vp.x, vp.y));
                            w[j] = half2_bits(q.x, q.y);
                        }
                        __syncwarp();
                        tmem_store16(t_p + 16 * c, w);
                    }
                    sum += s2.x + s2.y;
                    mids += m2.x + m2.y;
                    tc_wait_st();
                };
                if (busy) {
                    uint32_t see0 = s_valid[stage][2 * x], see1 = s_valid[stage][2 * x + 1];
                    const float2 la = s_level[stage][2 * x], lb = s_level[stage][2 * x + 1];
                    const float top = fmaxf(la.x, lb.x);
                    if ((see0 & see1) == 0xffffffffu && pos0 + 64 <= prefix && top - fminf(la.y, lb.y) <= kWideSpread) {
                        unit(std::true_type(), see0, see1, top);
                    } else {
                        // bits first .. first + 31 of the row's nodes, ones below 0 (wd is -1 for a negative first)
                        auto nodes = [&](int first) {
                            if (first <= -32) return 0xffffffffu;
                            const int wd = first >> 5;
                            const uint32_t lo = wd < 0 ? 0xffffffffu : wd * 32 < P.n_nodes ? s_seen[r][wd] : 0u;
                            const uint32_t hi = (wd + 1) * 32 < P.n_nodes ? s_seen[r][wd + 1] : 0u;
                            return __funnelshift_r(lo, hi, first & 31);
                        };
                        unit(std::false_type(), see0 & nodes(pos0 - prefix), see1 & nodes(pos0 + 32 - prefix), top);
                    }
                } else {
                    warp_arrive(b_read + 8 * x, lane);
                    // (no rows, but no running ahead either: an arrival must not count for a unit that others are still at)
                    if (n > 0) wide_wait(b_o + 8 * x, (n - 1) & 1, dead, P.wait_polls);
                }
                if (x == 1 && k == k0 && it > 0) wide_wait(b_free, (it - 1) & 1, dead, P.wait_polls);   // A has read O of the item before
                tc_before_sync();
                warp_arrive(b_p + 8 * x, lane);
                warp_arrive(b_empty + 8 * stage, lane);           // the parameters are read
                if (++stage == kWideStages) { stage = 0; phase ^= 1; }
            }
            // ---- the end of the item: B hands its rows to A
            wide_wait(b_o + 8 * x, (n - 1) & 1, dead, P.wait_polls);
            tc_after_sync();
            if (x == 1) {
                // (s_other is free: A has passed b_free for the item before, see above)
                s_other[r] = make_float4(ref, sum, mids, 0.f);
                tc_before_sync();
                warp_arrive(b_merge, lane);
            } else {
                wide_wait(b_merge, it & 1, dead, P.wait_polls);
                tc_after_sync();
                if (busy) {
                    const float4 other = s_other[r];
                    const float m = fmaxf(ref, other.x);
                    const float fa = att_factor(ref, sum, m), fb = att_factor(other.x, other.y, m);
                    const float z = fmaf(fa, mids, fb * other.z);
                    float l = fmaf(fa, sum, fb * other.y);
                    if (*dead) l = __int_as_float(0x7fffffff);
                    const float inv = l == 0.f ? 0.f : 1.f / l;   // (nothing seen: zeros)
                    const long long out = b * P.o_seq + node * P.o_node + h * P.o_head;
                    float *part = P.part + static_cast<long long>(2 * blockIdx.x + (k0 > 0 ? 0 : 1)) * part_floats(kWideRows, D);
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16], ob[16];
                        __syncwarp();
                        tmem_load16(t_o + 16 * c, o);
                        tmem_load16(t_o + D + 16 * c, ob);
                        if (row < P.n_rows) {
#pragma unroll
                            for (int i = 0; i < 16; i += 8) {     // eight columns: one word's codes, in the operands' order
                                float v[8];
#pragma unroll
                                for (int p = 0; p < 8; ++p)
                                    v[(p >> 1) + 4 * (p & 1)] = fmaf(fmaf(fa, __uint_as_float(o[i + p]), fb * __uint_as_float(ob[i + p])),
                                                                     (p & 2) ? 1048576.f : 16777216.f, z);
                                if (whole) {
#pragma unroll
                                    for (int e = 0; e < 8; ++e) v[e] *= inv;
                                    if (P.o_vec) {
                                        *reinterpret_cast<uint4 *>(static_cast<char *>(P.out) + 2 * (out + 16 * c + i)) = pack_elems<DT>(v);
                                    } else {
#pragma unroll
                                        for (int e = 0; e < 8; ++e) store_elem<DT>(P.out, out + 16 * c + i + e, v[e]);
                                    }
                                } else {
                                    float4 *to = reinterpret_cast<float4 *>(part + r * D + 16 * c + i);
                                    to[0] = make_float4(v[0], v[1], v[2], v[3]);
                                    to[1] = make_float4(v[4], v[5], v[6], v[7]);
                                }
                            }
                        }
                    }
                    if (row < P.n_rows) {
                        if (!whole) {
                            part[kWideRows * D + r] = m;
                            part[kWideRows * (D + 1) + r] = l;
                        } else if (P.lse) {
                            P.lse[(static_cast<long long>(b) * P.n_nodes + node) * P.n_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
                        }
                    }
                }
                __syncwarp();
                tc_before_sync();
                warp_arrive(b_free, lane);
            }
            ++it;
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
