// Attention of chunks with many rows per key/value head: two tiles of 128 rows a block on the tcgen05 tensor cores.
#pragma once

#include "mcsd_attend_wide.cuh"
#include "mcsd_chunk.cuh"

namespace mcsd {

#define MCSD_INLINE __attribute__((always_inline))

constexpr int kChunkRows = 256;                     // rows of a block: tiles A and B of 128
constexpr int kChunkThreads = 640;                  // 8 softmax warps, 8 decoding warps, 2 that issue (and 2 beside them)
constexpr float kChunkHead = 4.f;                   // log2 of a row's largest weight when its reference is set
constexpr float kChunkMost = 2048.f;                // sum of the weights of half a unit above which the reference moves (half holds 2^15, and 16 times this)
template <int D> constexpr int kChunkAhead = D == 128 ? 1 : 3;         // units whose codes are on their way to shared memory
constexpr int kChunkParams = 4;                     // units whose parameters are kept
template <int D> constexpr int kChunkSmem = 1024 + 6 * kWideTile<D> + kChunkParams * kAttUnit * 8 + kChunkAhead<D> * kAttUnit * (D + 16);

// D (tensor memory) (+)= A (shared memory, 128 rows x 16) * B (shared memory), halves in, float32 out.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a_low, uint32_t b_low, uint32_t high, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}"
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(high), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}

#define MCSD_R16(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7]), \
    "=r"(v[i + 8]), "=r"(v[i + 9]), "=r"(v[i + 10]), "=r"(v[i + 11]), "=r"(v[i + 12]), "=r"(v[i + 13]), "=r"(v[i + 14]), "=r"(v[i + 15])
// 64 columns of this warp's 32 lanes, lane i of the warp row i.
__device__ __forceinline__ void tmem_load64(uint32_t at, uint32_t (&v)[64]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
                 "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
                 "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"   // (in the same statement: the registers hold nothing before it)
                 : MCSD_R16(v, 0), MCSD_R16(v, 16), MCSD_R16(v, 32), MCSD_R16(v, 48) : "r"(at) : "memory");
}
#undef MCSD_R16

// Four codes of a value row as numbers: two nibbles of every byte pair, `odd` the higher ones. 1024 + c (or 1024 + 16 c) has the code in
// its lowest bits; both lines below are exact, the last rounds scale (c - 8) + mid once.
template <bool odd>
__device__ __forceinline__ __half2 value_pair(uint32_t w, __half2 scale, __half2 mid)
{
    const uint32_t bits = (w & (odd ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;
    const __half2 c = *reinterpret_cast<const __half2 *>(&bits);
    const __half2 n = odd ? __hfma2(c, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hsub2(c, __float2half2_rn(1032.f));
    return __hfma2(n, scale, mid);
}

// One CTA per SM. A block is up to 256 rows (tokens x query heads of one key head), 128 in each of the tiles A and B; a unit is 128 keys, in
// two halves of 64. A unit is decoded once for both tiles. Roles:
//   key warps (4)     codes come by cp.async AHEAD units before their use; one AND makes two of them subnormal halves (exact, c 2^-24), which
//                     go to shared memory as an operand. A key's scale and mid go there as float32 and are kept for kChunkParams units;
//   value warps (4)   scale (c - 8) + mid, rounded to half once: the product's other operand can have nothing left to apply;
//   issuing warps (2) one per tile: S = Q K^T of each half of a unit into its own 64 columns of tensor memory, O += P V with P over S;
//   softmax warps (8) one thread per row: s = ra (scale acc + (mid - 8 scale) rho), where rho is the row's sum of queries, so that K is exact
//                     (lse off by 9e-6 at most with fp16 queries, 7e-6 with bf16 ones; key_codes make it 3e-6 and 2e-6, and a call 3.5 % longer);
//                     weights 2^(s - ref), their sum in float32, and P to tensor memory.
// The maximum of a row is not formed for every unit. A row's reference is set in its first half unit (2^kChunkHead below its largest weight)
// and holds until a half unit's sum passes kChunkMost; then the half is done again with a maximum (careful), O scaled by the factor
// in tensor memory. Weights are rounded to half, relative to the largest one of the row so far: 2^-11 of each, or 2^-25 of 2^-kChunkHead where they are
// subnormal. For fp16 results, which show that, P has two parts (PARTS), the second what the first leaves: with the values' rounding 1.4 times
// the error of rounding the result, 1.55 without; bf16 results show neither. Values that half does not hold (beyond 65504, by scale and mid) are stored
// as a sixteenth and their weights are sixteen times as large; rows that are NaN or infinite are zeros in the operand and make
// the weights NaN where they are seen.
// While weights of one half are formed, the scores of the other are computed: all scores of a unit at once, P over them, took 1.72 instead of 1.45 ms
// (2048 tokens, 32 heads on 8 of 128 numbers, over 30011 rows), P apart from S with S given back early 1.48, parameters as pairs of halves 1.71.
// Keeping parameters for four units, so that a decoded tile is free once its products are done, took it from 1.45 to 1.36 ms.
// What bounds it: shared memory. A unit of 256 rows takes about 5800 cycles, of which its bandwidth has 2048 for broadcast loads of parameters by the softmax
// warps, 2048 for the operands of the products (Q, K and V; P comes from tensor memory) and 512 for the decoded tiles; beside that the
// chain softmax -> P V -> S of a half. With the parameters left out it would be 1.0 ms, without the exponentials or the decoding 1.19 each.
// Measured: 1.36 to 1.40 ms there, 770 to 745 TFLOP/s, 0.49 to 0.48 of the library's rate for large bf16 products; 64 numbers a head in fp16 1.52 ms (342).
template <int DT, int D>
__global__ void __launch_bounds__(kChunkThreads, 1)
chunk_wide_kernel(const __grid_constant__ ChunkParams P)
{
    constexpr int TILE = kWideTile<D>, RB = D / 2, AHEAD = kChunkAhead<D>;
    constexpr uint32_t kS = 0, kO = 256, kColumns = 512;                // S: 64 columns per tile and half of a unit's keys; P over the first 32 of them
    // Weights of one half each, or (where the result has half's precision, which the values' rounding takes its share of) with what that leaves.
    constexpr int PARTS = DT == MCSD_DTYPE_F16 ? 2 : 1;
    extern __shared__ unsigned char s_raw[];
    __shared__ __align__(8) unsigned long long s_bar[23];
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    // of a unit: keys that are there; values that are no numbers, or far from one
    __shared__ __align__(16) uint32_t s_valid[kChunkParams][4], s_bad[kChunkParams][4], s_far[kChunkParams][4];
    // Each warp goes over the CTA's blocks for itself; where it stands is kept here, since registers are short.
    __shared__ ChunkRows::Walk s_walk[kChunkThreads / 32];
    __shared__ AttItem s_item[kChunkThreads / 32];
    __shared__ int s_any;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    unsigned char *base = s_raw + ((1024 - (smem_u32(s_raw) & 1023)) & 1023);
    unsigned char *s_q = base, *s_k = base + 2 * TILE, *s_v = base + 4 * TILE;  // Q of both tiles, two stages each of keys and values
    float4 *s_param = reinterpret_cast<float4 *>(base + 6 * TILE);              // [kChunkParams][64 pairs of keys]
    unsigned char *s_codes = reinterpret_cast<unsigned char *>(s_param + kChunkParams * (kAttUnit / 2));   // [decoding warps][AHEAD]{codes, parameters}

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = smem_u32(s_bar);
    const uint32_t b_kfull = bars, b_kempty = bars + 16, b_vfull = bars + 32, b_vempty = bars + 48, b_ready = bars + 64, b_s = bars + 80,
                   b_p = bars + 112, b_o = bars + 144, b_end = bars + 176;      // b_s, b_p, b_o: [tile][half of the keys]
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_kfull + 8 * i, 4);          // (arrivals of warps)
            mbar_init(b_kempty + 8 * i, 2);         // (the products of both tiles)
            mbar_init(b_vfull + 8 * i, 4);
            mbar_init(b_vempty + 8 * i, 2);
            mbar_init(b_ready + 8 * i, 4 + P.test_extra);       // (0 but in a test of the expiry path: arrivals that never come)
            for (int h = 0; h < 2; ++h) {
                mbar_init(b_s + 16 * i + 8 * h, 2);             // (the products, and the warp that has seen the keys' parameters)
                mbar_init(b_p + 16 * i + 8 * h, 4);
                mbar_init(b_o + 16 * i + 8 * h, 1);
            }
        }
        mbar_init(b_end, 2);
        fence_mbar_init();
        s_dead = 0;
    }
    if (warp == 16) tmem_alloc(smem_u32(&s_tmem), kColumns);
    if (tid == 0) chunk_join_none(P);
    if (warp == 17) {
        ChunkRows::Walk walk;
        const bool any = walk.begin(P, lane);
        if (lane == 0) s_any = any;
        if (any && lane < kChunkThreads / 32) s_walk[lane] = walk;
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    constexpr uint32_t tmem = 0;
    volatile int *dead = &s_dead;
    if (s_tmem != tmem) *dead = 1;                  // (cannot be: all columns are this CTA's)

    const int ps = 1 << P.c.page_shift;
    // Every role goes over the same blocks.
    auto for_items = [&](auto f) MCSD_INLINE {
        if (!s_any) return;
        for (;;) {
            int more = 0;
            __syncwarp();
            if (lane == 0) {
                more = s_walk[warp].template next<kChunkRows>(P, lane, s_item[warp]);
            }
            if (!__shfl_sync(0xffffffffu, more, 0)) break;
            __syncwarp();
            f(s_item[warp]);
        }
    };
    // Units of a block that tile x has work in: those its last row sees (its rows' tokens end before the block's where it is tile A).
    auto tile_units = [&](const AttItem &it, int x) MCSD_INLINE {
        const int row = min(it.row0 + 128 * x + 127, it.rows - 1);
        if (it.row0 + 128 * x >= it.rows) return 0;
        const long long sees = static_cast<long long>(it.tail) + row / P.group - it.row0 / P.group;
        return chunk_units(static_cast<int>(min(sees, static_cast<long long>(it.len))));
    };

    if (warp >= 8 && warp < 16) {
        // ------------------------------------------------------------ decoding
        regs_down<56>();
        // Four warps have the key rows of every unit, four the value rows, 32 each: lane by lane, 16 bytes of codes at
        // 16 (lane + 32 i) of the rows of sixteen keys, so that a load is contiguous, and the parameters of key `lane`.
        constexpr int CH = RB / 16;                 // 16-byte chunks of a row: 2 or 4
        const int which = (warp >> 2) & 1, key0 = (warp & 3) * 32;       // which: 0 key rows, 1 value rows
        const int c = lane % CH;
        const uint32_t full = which ? b_vfull : b_kfull, empty = which ? b_vempty : b_kempty;
        constexpr int SLOT = 32 * (RB + 8);         // codes, parameters of these rows, parameters of the values (key warps)
        unsigned char *ring = s_codes + (warp & 7) * AHEAD * SLOT;
        int stage = 0, keep = 0;                    // stage of the unit, and where its parameters are kept
        uint32_t phase = 1;                         // (the first round of stages is free)
        for_items([&](const AttItem &it) MCSD_INLINE {
            const int len = it.len, k1 = it.k1;
            const int32_t *table = P.table + it.b * P.ld_table;
            const unsigned char *pool = P.c.pages + static_cast<long long>(it.head) * kv_block_bytes(D, ps);
            // page of this lane's half (lanes 0..15: the first sixteen keys)
            auto page_of = [&](int k) MCSD_INLINE {
                const int pos = k * kAttUnit + key0 + (lane & 16);
                return k < k1 && pos < len ? __ldg(table + (pos >> P.c.page_shift)) : -1;
            };
            uint32_t there = 0u;                    // bit `slot`: this lane's key of that unit is in the cache
            int page = -1;                          // of the unit asked for next
            auto issue = [&](int unit, int slot) MCSD_INLINE {
                const int pos = unit * kAttUnit + key0 + lane;
                unsigned char *to = ring + slot * SLOT;
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
                    if (ok) {
                        const unsigned char *src = pool + page * P.c.page_stride + ps * D + (pos & (ps - 1)) * 4;
                        cp_async4(to + 32 * RB + lane * 4, src + which * ps * 4);
                        if (which == 0) cp_async4(to + 32 * RB + 128 + lane * 4, src + ps * 4);
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            int pages[AHEAD + 1];
#pragma unroll
            for (int i = 0; i <= AHEAD; ++i) pages[i] = page_of(it.k0 + i);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                page = pages[i];
                issue(it.k0 + i, i);
            }
            page = pages[AHEAD];
            int slot = 0;
            for (int k = it.k0; k < k1; ++k) {
                asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
                const unsigned char *from = ring + slot * SLOT;
                // what this lane copied itself: its codes, and the parameters of its key
                uint4 code[CH];
#pragma unroll
                for (int i = 0; i < CH; ++i) code[i] = *reinterpret_cast<const uint4 *>(from + i * 512 + lane * 16);
                const bool mine = (there >> slot) & 1u;
                const uint32_t raw = *reinterpret_cast<const uint32_t *>(from + 32 * RB + lane * 4);
                const uint32_t raw_value = *reinterpret_cast<const uint32_t *>(from + 32 * RB + 128 + lane * 4);      // (of a key warp)
                issue(k + AHEAD, slot);
                page = page_of(k + AHEAD + 1);      // (in flight until the next unit is asked for)
                slot = slot == AHEAD - 1 ? 0 : slot + 1;
                wide_wait(empty + 8 * stage, phase, dead, P.wait_polls);
                const float2 p = mine ? __half22float2(*reinterpret_cast<const __half2 *>(&raw)) : make_float2(0.f, 0.f);
                // values that are numbers, and those that half may not hold (a row's ends, by the roundings of its scale and mid)
                const float2 pv = which == 0 && mine ? __half22float2(*reinterpret_cast<const __half2 *>(&raw_value)) : p;
                const bool sound = fabsf(pv.x) <= 65504.f && fabsf(pv.y) <= 65504.f;
                const uint32_t bad = __ballot_sync(0xffffffffu, mine && !sound);
                const uint32_t far = __ballot_sync(0xffffffffu, mine && sound && fmaf(8.f, fabsf(pv.x), fabsf(pv.y)) > 65000.f);
                unsigned char *tiles = (which ? s_v : s_k) + stage * TILE;
                auto place = [&](int i, int j) MCSD_INLINE {            // where 16 bytes of operands go: chunk i of the lane, its word j
                    const int key = key0 + (i / (CH / 2)) * 16 + (i % (CH / 2)) * (32 / CH) + lane / CH;
                    const int chunk = 4 * c + j;
                    return reinterpret_cast<uint4 *>(tiles + key * 128 + (chunk >> 3) * (kAttUnit * 128) + (((chunk & 7) ^ (key & 7)) << 4));
                };
                // (with four chunks a row, lanes 2 and 3 take their words in another order: no two lanes of eight meet in a bank)
                const bool turn = CH == 4 && (c & 2);
                auto word = [&](const uint4 &v, int j) MCSD_INLINE {
                    return j == 0 ? (turn ? v.z : v.x) : j == 1 ? (turn ? v.w : v.y) : j == 2 ? (turn ? v.x : v.z) : (turn ? v.y : v.w);
                };
                if (which == 0) {
                    // keys: codes as subnormal halves (one AND for two of them); scale and mid enter the scores in float32
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t w = word(code[i], j), y = w >> 8;
                            *place(i, turn ? j ^ 2 : j) = make_uint4(w & 0x000f000fu, w & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u);
                        }
                    const int key = key0 + lane;
                    float *par = reinterpret_cast<float *>(s_param + keep * (kAttUnit / 2) + (key >> 1)) + (key & 1);
                    par[0] = p.x * P.scale_part;
                    par[2] = fmaf(-8.f, p.x, p.y) * P.scale_part;
                    const uint32_t keys = __ballot_sync(0xffffffffu, mine);
                    if (lane == 0) { s_valid[keep][warp & 3] = keys; s_bad[keep][warp & 3] = bad; s_far[keep][warp & 3] = far; }
                } else {
                    // values: numbers in half, rounded once. Rows that are no numbers are zeros here (and marked); those that half may not hold
                    // are stored as a sixteenth, and their weights are sixteen times as large
                    uint32_t own = mine && sound ? raw : 0u;
                    if ((far >> lane) & 1u) own = half2_bits(p.x * 0.0625f, p.y * 0.0625f);
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const uint32_t both = __shfl_sync(0xffffffffu, own, (i / (CH / 2)) * 16 + (i % (CH / 2)) * (32 / CH) + lane / CH);
                        const __half2 h = *reinterpret_cast<const __half2 *>(&both), scale = __low2half2(h), mid = __high2half2(h);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t w = word(code[i], j), y = w >> 8;
                            const __half2 x[4] = {value_pair<false>(w, scale, mid), value_pair<true>(w, scale, mid), value_pair<false>(y, scale, mid),
                                            value_pair<true>(y, scale, mid)};
                            *place(i, turn ? j ^ 2 : j) = *reinterpret_cast<const uint4 *>(x);
                        }
                    }
                }
                fence_proxy_async();
                warp_arrive(full + 8 * stage, lane);
                if (++stage == 2) { stage = 0; phase ^= 1; }
                keep = (keep + 1) % kChunkParams;
            }
        });
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= 16) {
        // ------------------------------------------------------------ issuing
        regs_down<32>();
        const int x = warp - 16;                    // the tile it issues for
        if (x < 2) {
            int stage = 0, ahead = 0;               // stages of the unit whose weights are next, and of the one whose scores are
            uint32_t phase = 0, ahead_phase = 0, n = 0, items = 0;      // n: units of this tile so far
            const uint32_t q_at = tc_operand(smem_u32(s_q) + x * TILE, 16);
            // Scores of half h of the unit at `ahead`, the tile's unit m: over the weights of the unit before, whose products are done first.
            auto scores = [&](int h, uint32_t m) MCSD_INLINE {
                if (h == 0) wide_wait(b_kfull + 8 * ahead, ahead_phase, dead, P.wait_polls);
                if (m > 0) wide_wait(b_o + 16 * x + 8 * h, (m - 1) & 1, dead, P.wait_polls);
                tc_after_sync();
                const uint32_t at = tc_operand(smem_u32(s_k) + ahead * TILE + h * 64 * 128, 16);
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    const uint32_t off = (s >> 2) * (kAttUnit * 128 / 16) + (s & 3) * 2;
                    tc_mma_ss(tmem + kS + 128 * x + 64 * h, q_at + off, at + off, kOperandHigh, tc_shape(64, false), s > 0);
                }
                tc_commit(b_s + 16 * x + 8 * h);
                warp_arrive(b_s + 16 * x + 8 * h, lane);
                if (h == 1) {
                    tc_commit(b_kempty + 8 * ahead);
                    if (++ahead == 2) { ahead = 0; ahead_phase ^= 1; }
                }
            };
            for_items([&](const AttItem &it) MCSD_INLINE {
                const int k0 = it.k0, k1 = it.k1, mine = min(tile_units(it, x), k1);
                if (k0 < mine) {                    // (a tile without work has no queries either: nobody may run ahead of this barrier)
                    wide_wait(b_ready + 8 * x, items & 1, dead, P.wait_polls);
                    ++items;
                    scores(0, n);
                    scores(1, n);
                }
                for (int k = k0; k < k1; ++k) {
                    const bool work = k < mine;
                    if (!work) {                    // (a tile's units are the first ones: nothing is ahead here)
                        wide_wait(b_kfull + 8 * ahead, ahead_phase, dead, P.wait_polls);
                        tc_commit(b_kempty + 8 * ahead);
                        if (++ahead == 2) { ahead = 0; ahead_phase ^= 1; }
                    }
                    wide_wait(b_vfull + 8 * stage, phase, dead, P.wait_polls);
                    if (work) {
                        const uint32_t at = tc_operand(smem_u32(s_v) + stage * TILE, kAttUnit * 128);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            wide_wait(b_p + 16 * x + 8 * h, n & 1, dead, P.wait_polls);
                            tc_after_sync();
#pragma unroll
                            for (int s = 0; s < 4 * PARTS; ++s)
                                tc_mma(tmem + kO + D * x, tmem + kS + 128 * x + 64 * h + 8 * s, at + (4 * h + s % 4) * (16 * 128 / 16), kOperandHigh, tc_shape(D, true),
                                       k > k0 || h > 0 || s > 0);
                            tc_commit(b_o + 16 * x + 8 * h);
                            if (h == 1) tc_commit(b_vempty + 8 * stage);
                            if (k + 1 < mine) scores(h, n + 1);
                        }
                        ++n;
                    } else {
                        tc_commit(b_vempty + 8 * stage);
                    }
                    if (++stage == 2) { stage = 0; phase ^= 1; }
                }
            });
            // What was issued, by both warps, ends before its memory is given back. (Where no wait expires, the softmax groups have
            // waited for the products already; where one does, it may be the last of all, after this warp is through.)
            tc_commit(b_end);
            for (uint32_t i = 0; i < kWaitPolls && !__all_sync(0xffffffffu, mbar_try_wait(b_end, 0)); ++i) {}
        }
    } else {
        // ------------------------------------------------------------ softmax
        regs_up<168>();
        const int x = warp >> 2;                    // tile
        const int r = tid & 127;                    // row of the tile = lane of tensor memory
        const uint32_t mine = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + mine + kS + 128 * x, t_o = tmem + mine + kO + D * x;
        int keep = 0;                               // where the unit's parameters are kept
        uint32_t n = 0;
        for_items([&](const AttItem &it) MCSD_INLINE {
            if (tid == 0) chunk_join_note(P, it);
            const int row = it.row0 + 128 * x + r;
            const bool live = row < it.rows;
            const int units = tile_units(it, x);
            // positions this row sees (a row that is none sees what the last one does), and those that all rows of the tile see
            const int token = min(row, it.rows - 1) / P.group - it.row0 / P.group;
            const int sees = static_cast<int>(min(static_cast<long long>(it.tail) + token, static_cast<long long>(it.len)));
            const int all = static_cast<int>(min(static_cast<long long>(it.tail) + min(it.row0 + 128 * x, it.rows - 1) / P.group - it.row0 / P.group, static_cast<long long>(it.len)));
            float rho = 0.f, ra = 0.f;              // score in log2 units: ra (scale acc + (mid - 8 scale) rho), ra a power of two
            const int k0 = it.k0, k1 = it.k1;
            const bool any = k0 < units;            // (of the tile)
            if (any) {
                // Q to shared memory, scaled by a power of two to the top of half's range (and to a positive softmax scale), in the order that
                // the ANDs of the keys give. The rows come side by side, sixteen bytes a lane, to where their operands go; then each thread
                // turns its own, sixteen bytes at a time.
                constexpr int CR = D / 8;           // 16-byte chunks of a row
                auto place = [&](int rr, int c) MCSD_INLINE { return s_q + x * TILE + rr * 128 + (c >> 3) * (kAttUnit * 128) + (((c & 7) ^ (rr & 7)) << 4); };
                const long long at = live ? ChunkRows::q_at(P, it, row) : -1;
                if (P.q_vec) {
#pragma unroll 4
                    for (int i = 0; i < CR; ++i) {
                        const int rr = i * (32 / CR) + lane / CR, c = lane % CR;
                        const long long from = __shfl_sync(0xffffffffu, at, rr);
                        if (from >= 0) cp_async16(smem_u32(place((warp & 3) * 32 + rr, c)), static_cast<const char *>(P.q) + 2 * (from + 8 * c));
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    __syncwarp();
                } else if (live) {
                    const unsigned short *src = static_cast<const unsigned short *>(P.q) + at;
#pragma unroll 1
                    for (int c = 0; c < CR; ++c)
                        *reinterpret_cast<uint4 *>(place(r, c)) =
                            make_uint4(src[8 * c] | src[8 * c + 1] << 16, src[8 * c + 2] | src[8 * c + 3] << 16,
                                       src[8 * c + 4] | src[8 * c + 5] << 16, src[8 * c + 6] | src[8 * c + 7] << 16);
                }
                auto chunk = [&](int c) MCSD_INLINE { return live ? *reinterpret_cast<const uint4 *>(place(r, c)) : make_uint4(0u, 0u, 0u, 0u); };
                uint32_t big = 0u;                  // largest magnitudes of two numbers
#pragma unroll 4
                for (int c = 0; c < CR; ++c) {
                    const uint4 v = chunk(c);
                    big = Elem<DT>::mx(Elem<DT>::mx(big, v.x & 0x7fff7fffu), Elem<DT>::mx(v.y & 0x7fff7fffu, Elem<DT>::mx(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
                }
                const float most = Elem<DT>::max_final(big);
                int e = most > 0.f ? static_cast<int>(__float_as_uint(most) >> 23) - 126 : 0;
                e = max(min(e, 112), -110);
                const float up = __int_as_float((127 + 15 - e) << 23) * (P.scale < 0.f ? -1.f : 1.f);
                ra = ldexpf(1.f, P.scale_power + e - 15 + 24);
                float2 sum = make_float2(0.f, 0.f);
                const float2 f0 = make_float2(up, up), f1 = make_float2(up * 0.0625f, up * 0.0625f);
#pragma unroll 2
                for (int c = 0; c < CR; ++c) {      // eight numbers, one word of codes
                    float v[8];
                    Elem<DT>::unpack(chunk(c), v);
                    uint32_t out[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 pair = make_float2(v[i], v[i + 4]);
                        sum = add2(sum, pair);
                        const float2 q = __fmul2_rn(pair, i & 1 ? f1 : f0);
                        out[i] = half2_bits(q.x, q.y);
                    }
                    *reinterpret_cast<uint4 *>(place(r, c)) = make_uint4(out[0], out[1], out[2], out[3]);
                }
                rho = (sum.x + sum.y) * up * 5.9604644775390625e-8f;            // 2^-24
                fence_proxy_async();
                tc_before_sync();
                warp_arrive(b_ready + 8 * x, lane);
            }
            float ref = kNoTop, sum = 0.f;
            for (int k = k0; k < k1; ++k) {
                if (k < units) {
                    const float4 *par = s_param + keep * (kAttUnit / 2);
                    auto rest = [](float2 p, uint32_t w) MCSD_INLINE {     // of two weights beyond their halves
                        const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&w));
                        return half2_bits(p.x - h.x, p.y - h.y);
                    };
                    // One half of the unit's keys, where every row of the tile sees them and nothing is odd about the values: the
                    // weights with the reference as it is; false (and nothing stored) should their sum be too large for half.
                    auto swift = [&](int h) MCSD_INLINE {
                        uint32_t acc[64], w[32 * PARTS];
                        tmem_load64(t_s + 64 * h, acc);
                        float2 s2 = make_float2(0.f, 0.f);
                        const float rr = rho * ra;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float4 kp = par[32 * h + j];
                            const float2 a = __fmul2_rn(make_float2(kp.x, kp.y), make_float2(ra, ra));
                            const float2 m = fma2(make_float2(kp.z, kp.w), make_float2(rr, rr), make_float2(-ref, -ref));
                            const float2 e = fma2(make_float2(__uint_as_float(acc[2 * j]), __uint_as_float(acc[2 * j + 1])), a, m);
                            const float2 p = make_float2(ex2f(e.x), ex2f(e.y));
                            s2 = add2(s2, p);
                            w[j] = half2_bits(p.x, p.y);
                            if constexpr (PARTS == 2) w[32 + j] = rest(p, w[j]);
                        }
                        if (__any_sync(0xffffffffu, s2.x + s2.y > kChunkMost)) return false;
                        sum += s2.x + s2.y;
#pragma unroll
                        for (int c = 0; c < 2 * PARTS; ++c) tmem_store16(t_s + 64 * h + 16 * c, *reinterpret_cast<const uint32_t(*)[16]>(w + 16 * c));
                        return true;
                    };
                    // The same wherever the first does not do: the largest score, the reference moved where that leaves it by too much, then
                    // the weights, sixteen keys at a time. see0, see1: the keys that this row sees; bad, far: values that are no numbers (their
                    // rows are none), or far from one.
                    auto careful = [&](int h, uint32_t see0, uint32_t see1) MCSD_INLINE {
                        const float4 *at = par + 32 * h;
                        float most = -INFINITY;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t see = (c < 2 ? see0 : see1) >> (16 * (c & 1));
                            uint32_t acc[16];
                            __syncwarp();
                            tmem_load16(t_s + 64 * h + 16 * c, acc);
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const float4 kp = at[8 * c + j];
                                const float2 z = fma2(make_float2(__uint_as_float(acc[2 * j]), __uint_as_float(acc[2 * j + 1])), make_float2(kp.x, kp.y),
                                                      __fmul2_rn(make_float2(kp.z, kp.w), make_float2(rho, rho)));
                                if ((see >> (2 * j)) & 1u) most = fmaxf(most, z.x);
                                if ((see >> (2 * j + 1)) & 1u) most = fmaxf(most, z.y);
                            }
                        }
                        const float high = most * ra - kChunkHead;
                        const bool move = high - ref > kNarrowSlack;            // (a difference that is exact, however large the two are)
                        if (__any_sync(0xffffffffu, move)) {
                            const float now = move ? high : ref;
                            const float f = ex2f(ref - now);
                            ref = now;
                            sum *= f;
                            if (k > k0 || h > 0) {
                                // the product of the half before is done (those before that are: these scores came after them)
                                wide_wait(b_o + 16 * x + 8 * (h ^ 1), (h == 0 ? n - 1 : n) & 1, dead, P.wait_polls);
                                tc_after_sync();
#pragma unroll 1
                                for (int c = 0; c < D / 16; ++c) {
                                    uint32_t o[16];
                                    __syncwarp();
                                    tmem_load16(t_o + 16 * c, o);
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                    tmem_store16(t_o + 16 * c, o);
                                }
                            }
                        }
                        float2 s2 = make_float2(0.f, 0.f);
                        // (What is stored lies over scores that are read: of weights in two parts, over all of them.)
                        constexpr int PER = PARTS == 2 ? 64 : 16;
#pragma unroll 1
                        for (int c = 0; c < 64 / PER; ++c) {
                            const int first = PER * c, word = 2 * h + (first >> 5);
                            uint32_t acc[PER], w[PER / 2 * PARTS];
                            __syncwarp();
                            if constexpr (PARTS == 2) tmem_load64(t_s + 64 * h, acc);
                            else tmem_load16(t_s + 64 * h + first, acc);
#pragma unroll
                            for (int j = 0; j < PER / 2; ++j) {
                                const int shift = (first & 31) + 2 * j & 31, more = j >> 4;
                                const uint32_t see = ((first >> 5) + more ? see1 : see0) >> shift;
                                const uint32_t far = s_far[keep][word + more] >> shift, bad = see & s_bad[keep][word + more] >> shift;
                                const float4 kp = at[first / 2 + j];
                                // (the same numbers as above, and their products with ra are exact: none is above its reference by more than the
                                // slack, however large a step of the scores is)
                                const float2 z = fma2(make_float2(__uint_as_float(acc[2 * j]), __uint_as_float(acc[2 * j + 1])), make_float2(kp.x, kp.y),
                                                      __fmul2_rn(make_float2(kp.z, kp.w), make_float2(rho, rho)));
                                const float2 e = fma2(z, make_float2(ra, ra), make_float2(-ref, -ref));
                                float2 p = make_float2(see & 1u ? ex2f(e.x) : 0.f, see & 2u ? ex2f(e.y) : 0.f);
                                s2 = add2(s2, p);
                                if (far & 1u) p.x *= 16.f;
                                if (far & 2u) p.y *= 16.f;
                                if (bad & 1u) p.x = __int_as_float(0x7fffffff);
                                if (bad & 2u) p.y = __int_as_float(0x7fffffff);
                                w[j] = half2_bits(p.x, p.y);
                                if constexpr (PARTS == 2) w[PER / 2 + j] = rest(p, w[j]);
                            }
                            if constexpr (PARTS == 2) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) tmem_store16(t_s + 64 * h + 16 * i, *reinterpret_cast<const uint32_t(*)[16]>(w + 16 * i));
                            } else {
                                tmem_store8(t_s + 64 * h + first / 2, w);
                            }
                        }
                        sum += s2.x + s2.y;
                    };
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        wide_wait(b_s + 16 * x + 8 * h, n & 1, dead, P.wait_polls);
                        tc_after_sync();
                        const int pos0 = k * kAttUnit + 64 * h;
                        const uint32_t there0 = s_valid[keep][2 * h], there1 = s_valid[keep][2 * h + 1];
                        const uint32_t odd = s_bad[keep][2 * h] | s_bad[keep][2 * h + 1] | s_far[keep][2 * h] | s_far[keep][2 * h + 1];
                        const bool plain = (there0 & there1) == 0xffffffffu && odd == 0u && pos0 + 64 <= all;
                        if (!plain || (k == k0 && h == 0) || !swift(h)) {       // (at first there is no reference)
                            auto first = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };
                            careful(h, there0 & first(sees - pos0), there1 & first(sees - pos0 - 32));
                        }
                        tc_wait_st();
                        tc_before_sync();
                        warp_arrive(b_p + 16 * x + 8 * h, lane);
                    }
                    ++n;
                }
                // (what is kept of a unit is written over four units later, when this tile's products of the one after it are through)
                keep = (keep + 1) % kChunkParams;
            }
            // ---- the end of the block
            if (any) {
                wide_wait(b_o + 16 * x, (n - 1) & 1, dead, P.wait_polls);
                wide_wait(b_o + 16 * x + 8, (n - 1) & 1, dead, P.wait_polls);
            }
            tc_after_sync();
            float l = sum;
            if (*dead) l = __int_as_float(0x7fffffff);
            const float inv = l == 0.f ? 0.f : 1.f / l;         // (nothing seen: zeros)
            const int at_row = 128 * x + r;
            float *part = P.part + att_slot(it.k0) * part_floats(kChunkRows, D);
            // The rows of a warp go through its part of the queries' memory (which nobody reads any more), so that they leave
            // side by side: 32 numbers of every row at a time as float32, or all of them in their type.
            unsigned char *own = s_q + x * TILE + (warp & 3) * 32 * 128;
            constexpr int CR = D / 8;               // 16-byte chunks of a row in its type
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                __syncwarp();
                tmem_load32(t_o + 32 * c, o);
#pragma unroll
                for (int i = 0; i < 4; ++i) {       // eight columns: one word's codes, in the operands' order
                    float v[8];
#pragma unroll
                    for (int p = 0; p < 8; ++p) v[(p >> 1) + 4 * (p & 1)] = any ? __uint_as_float(o[8 * i + p]) : 0.f;
                    if (it.whole) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= inv;
                        const int cc = 4 * c + i;
                        *reinterpret_cast<uint4 *>(own + lane * 128 + (cc >> 3) * (kAttUnit * 128) + (((cc & 7) ^ (lane & 7)) << 4)) = pack_elems<DT>(v);
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            *reinterpret_cast<float4 *>(own + lane * 128 + (((2 * i + e) ^ (lane & 7)) << 4)) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                    }
                }
                if (!it.whole) {
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int rr = 4 * i + (lane >> 3), grow = 128 * x + (warp & 3) * 32 + rr;
                        if (it.row0 + grow < it.rows)
                            *reinterpret_cast<float4 *>(part + grow * D + 32 * c + 4 * (lane & 7)) = *reinterpret_cast<const float4 *>(own + rr * 128 + (((lane & 7) ^ (rr & 7)) << 4));
                    }
                }
            }
            if (it.whole) {
                const long long row_at = live ? ChunkRows::out_at(P, it, row) : -1;
                __syncwarp();
#pragma unroll 4
                for (int i = 0; i < CR; ++i) {
                    const int rr = i * (32 / CR) + lane / CR, c = lane % CR;
                    const long long first = __shfl_sync(0xffffffffu, row_at, rr), at = first + 8 * c;
                    if (first >= 0) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(own + rr * 128 + (c >> 3) * (kAttUnit * 128) + (((c & 7) ^ (rr & 7)) << 4));
                        if (P.o_vec) {
                            *reinterpret_cast<uint4 *>(static_cast<char *>(P.out) + 2 * at) = v;
                        } else {
                            unsigned short *to = static_cast<unsigned short *>(P.out) + at;
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 8; ++e) to[e] = static_cast<unsigned short>(w[e >> 1] >> (16 * (e & 1)));
                        }
                    }
                }
            }
            if (live) {
                if (!it.whole) {
                    part[kChunkRows * D + at_row] = ref;
                    part[kChunkRows * (D + 1) + at_row] = l;
                } else if (P.lse) {
                    P.lse[ChunkRows::lse_at(P, it, row)] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
                }
            }
            __syncwarp();
            tc_before_sync();
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
