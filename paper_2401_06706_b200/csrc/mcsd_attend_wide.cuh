// Tree attention for many rows per key/value head: 128 rows a block on the tcgen05 tensor cores.
#pragma once

#include "mcsd_attend.cuh"

namespace mcsd {

constexpr int kWideRows = 128, kWideThreads = 512;  // two groups of softmax warps, one of decoding warps, one that issues
template <int D> constexpr int kWideTile = kAttUnit * D * 2;                       // bytes of a decoded tile of keys or values
template <int D> constexpr int kWideMerge = kWideRows * (D + 4) * 4;
template <int D> constexpr int kWideSmem = 1024 + 4 * kWideTile<D> + 2 * kAttUnit * 16 + kWideMerge<D> + kWideRows * (MCSD_MAX_NODES / 32) * 4;

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
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D (tensor memory) (+)= A (tensor memory, 128 rows x 16) * B (shared memory, described), halves in, float32 out.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
#define MCSD_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define MCSD_W8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// Sixteen columns of this warp's 32 lanes, lane i of the warp row i.
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
// row's index mod 8 (1024-byte groups of eight rows): `lead` is the distance to the next 64 numbers of the
// contiguous side where that side is not the summed one.
__device__ __forceinline__ uint64_t tc_operand(uint32_t at, uint32_t lead) {
    return static_cast<uint64_t>((at & 0x3ffffu) >> 4) | static_cast<uint64_t>(lead >> 4) << 16 | static_cast<uint64_t>(1024 >> 4) << 32 |
           1ull << 46 | 2ull << 61;
}
// 128 x n, half operands, float32 result; `outer`: B's contiguous side is n, not the summed one.
__host__ __device__ constexpr uint32_t tc_shape(int n, bool outer) {
    return 1u << 4 | (outer ? 1u << 16 : 0u) | static_cast<uint32_t>(n >> 3) << 17 | static_cast<uint32_t>(kWideRows >> 4) << 24;
}

// Registers per thread of the groups of four warps: the kernel is launched with 128 each, the group that
// issues and the one that decodes give away what the softmax groups take (2 x 176 + 112 + 48 = 4 x 128).
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Bounded wait of one of the roles below: false once it gives up, or another role has (every poll may
// suspend the thread for a microsecond, so the bound is a few seconds).
__device__ __forceinline__ bool wide_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
    for (uint32_t i = 0; i < kWaitPolls; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63) == 63 && *dead) return false;
    }
    *dead = 1;
    return false;
}
// The same for a whole warp, with one answer for all its lanes.
__device__ __forceinline__ bool wide_wait_warp(uint32_t bar, uint32_t parity, volatile int *dead) {
    return __all_sync(0xffffffffu, wide_wait(bar, parity, dead));
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// One CTA per SM, work cut as for the narrow kernel, in units of 128 keys. Roles:
//   decoding warps  (128 threads, one key each) take codes from global memory to operands in shared memory: a
//                   4-bit code becomes a subnormal half by one AND (see the narrow kernel), those of the values
//                   less 8, an exact subtraction; codes stay in the order the ANDs give them, which Q and the output undo;
//   issuing thread  S = Q K^T and O += P V by tcgen05.mma, Q and P from tensor memory, K and V from shared memory;
//   softmax groups  A and B (128 threads each, one row per thread) take keys 0..63 and 64..127 of every unit, each
//                   with maxima, sums and an O of its own, so that neither waits for the other: while one exponentiates,
//                   the tensor cores work for the other. They are joined at the end of an item.
// Scale and mid of a key enter the scores in float32; the weight p vscale is rounded to half once. The
// reference of a row's exponents is its maximum plus the exponent of the largest value scale, which keeps
// the weights in half's range whatever the scales are; it moves only when it is exceeded by 2^kNarrowSlack.
// Tensor memory (columns): S of A, S of B (64 each), O of A, O of B (D each), P of A, P of B (32 each), Q (D / 2).
template <int DT, int D>
__global__ void __launch_bounds__(kWideThreads, 1)
wide_kernel(const __grid_constant__ AttendParams P)
{
    constexpr int TILE = kWideTile<D>, RB = D / 2;
    constexpr uint32_t kS = 0, kO = 128, kP = 128 + 2 * D, kQ = 192 + 2 * D, kColumns = 512;
    extern __shared__ unsigned char s_raw[];
    __shared__ __align__(8) unsigned long long s_bar[13];
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    __shared__ uint32_t s_valid[2][4];              // keys of a stage that are there
    __shared__ float s_big[2][4];                   // largest value scale of 32 keys
    __shared__ float s_row[2][kWideRows];           // of a row: sum of q and log2 units, see below; then B's reference and sum
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    unsigned char *base = s_raw + ((1024 - (smem_u32(s_raw) & 1023)) & 1023);
    unsigned char *s_tiles = base;                                              // [2 stages][keys, values]
    float4 *s_param = reinterpret_cast<float4 *>(base + 4 * TILE);              // [2][64 pairs of keys]{key, value}
    float *s_merge = reinterpret_cast<float *>(base + 4 * TILE + 2 * kAttUnit * 16);
    uint32_t(*s_seen)[MCSD_MAX_NODES / 32] = reinterpret_cast<uint32_t(*)[MCSD_MAX_NODES / 32]>(
        base + 4 * TILE + 2 * kAttUnit * 16 + kWideMerge<D>);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = smem_u32(s_bar);
    const uint32_t b_full = bars, b_empty = bars + 16, b_s = bars + 32, b_p = bars + 48, b_o = bars + 64, b_ready = bars + 80,
                   b_free = bars + 88, b_merge = bars + 96;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_full + 8 * i, 128);
            mbar_init(b_empty + 8 * i, 9);          // the tensor cores, and eight softmax warps that read the parameters
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_p + 8 * i, 128);
            mbar_init(b_o + 8 * i, 1);
        }
        mbar_init(b_ready, 128);
        mbar_init(b_free, 128);
        mbar_init(b_merge, 128);
        fence_mbar_init();
        s_dead = 0;
    }
    if (warp == 12) tmem_alloc(smem_u32(&s_tmem), kColumns);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = s_tmem;
    volatile int *dead = &s_dead;

    const int ps = 1 << P.c.page_shift;
    const int items = P.c.n_heads * P.n_blocks;
    const long long total = att_units_before(P, P.batch, lane) * items;
    const long long per = max((total + P.n_ctas - 1) / P.n_ctas, 1LL);
    const long long u_begin = static_cast<long long>(blockIdx.x) * per, u_end = min(u_begin + per, total);

    // Every role goes over the same items; f(sequence, length, head, first row, first unit, last unit + 1, whole item).
    auto for_items = [&](auto f) {
        if (u_begin >= u_end) return;
        AttCursor cur = att_find(P, u_begin, items, lane);
        for (long long u = u_begin; u < u_end;) {
            const int item = static_cast<int>(cur.at / cur.units);
            const int k0 = static_cast<int>(cur.at - static_cast<long long>(item) * cur.units);
            const int k1 = static_cast<int>(min(static_cast<long long>(cur.units), k0 + (u_end - u)));
            const int head = item / P.n_blocks;
            if (!f(cur.b, cur.len, head, (item - head * P.n_blocks) * kWideRows, k0, k1, k0 == 0 && k1 == cur.units)) return;
            u += k1 - k0;
            cur.at += k1 - k0;
            if (u < u_end && cur.at >= static_cast<long long>(cur.units) * items) cur = att_find(P, u, items, lane);
        }
    };

    if (warp >= 8 && warp < 12) {
        // ------------------------------------------------------------ decoding
        regs_down<112>();
        const int key = tid - 256;
        uint32_t n = 0;                             // units so far
        for_items([&](int b, int len, int head, int, int k0, int k1, bool) {
            const int32_t *table = P.table + b * P.ld_table;
            const unsigned char *pool = P.c.pages + static_cast<long long>(head) * kv_block_bytes(D, ps);
            auto page_of = [&](int k) {
                const int pos = k * kAttUnit + key;
                return k < k1 && pos < len ? __ldg(table + (pos >> P.c.page_shift)) : -1;
            };
            struct Row { uint4 codes[2][RB / 16]; uint32_t param[2]; bool there; };
            auto fetch = [&](int k, int page, Row &r) {
                r.there = static_cast<unsigned>(page) < static_cast<unsigned>(P.c.n_pages);
                r.param[0] = r.param[1] = 0u;
#pragma unroll
                for (int i = 0; i < RB / 16; ++i) r.codes[0][i] = r.codes[1][i] = make_uint4(0u, 0u, 0u, 0u);
                if (r.there) {
                    const int row = (k * kAttUnit + key) & (ps - 1);
                    const unsigned char *block = pool + page * P.c.page_stride;
                    const uint4 *kc = reinterpret_cast<const uint4 *>(block + row * RB);
                    const uint4 *vc = reinterpret_cast<const uint4 *>(block + (ps + row) * RB);
                    const uint32_t *par = reinterpret_cast<const uint32_t *>(block + ps * D) + row;
#pragma unroll
                    for (int i = 0; i < RB / 16; ++i) { r.codes[0][i] = __ldg(kc + i); r.codes[1][i] = __ldg(vc + i); }
                    r.param[0] = __ldg(par);
                    r.param[1] = __ldg(par + ps);
                }
            };
            Row now, next;
            int page = page_of(k0);
            fetch(k0, page, now);
            page = page_of(k0 + 1);
            for (int k = k0; k < k1; ++k, ++n) {
                const int stage = n & 1;
                fetch(k + 1, page, next);           // (in flight while this unit is decoded)
                page = page_of(k + 2);
                if (n >= 2 && !wide_wait_warp(b_empty + 8 * stage, ((n >> 1) - 1) & 1, dead)) return false;
                // keys, then values: 16 bytes of codes are four 16-byte chunks of operands
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    unsigned char *tile = s_tiles + (2 * stage + which) * TILE + key * 128;
#pragma unroll
                    for (int i = 0; i < RB / 16; ++i) {
                        const uint32_t w[4] = {now.codes[which][i].x, now.codes[which][i].y, now.codes[which][i].z, now.codes[which][i].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t y = w[j] >> 8;
                            uint32_t h[4] = {w[j] & 0x000f000fu, w[j] & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u};
                            if (which) {            // less 8 (in units of 2^-24, the odd ones of 2^-20): exact
                                const uint32_t eight[2] = {0x00080008u, 0x00800080u};
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&h[q]), *reinterpret_cast<const __half2 *>(&eight[q & 1]));
                                    h[q] = *reinterpret_cast<const uint32_t *>(&d);
                                }
                            }
                            const int chunk = 4 * i + j;
                            *reinterpret_cast<uint4 *>(tile + (chunk >> 3) * (kAttUnit * 128) + (((chunk & 7) ^ (key & 7)) << 4)) =
                                make_uint4(h[0], h[1], h[2], h[3]);
                        }
                    }
                }
                // scale and mid - 8 scale of the key, scale and mid of the value, in pairs of keys
                const float2 kp = __half22float2(*reinterpret_cast<const __half2 *>(&now.param[0]));
                const float2 vp = __half22float2(*reinterpret_cast<const __half2 *>(&now.param[1]));
                float *par = reinterpret_cast<float *>(s_param + stage * kAttUnit + (key >> 1) * 2) + (key & 1);
                par[0] = kp.x;
                par[2] = fmaf(-8.f, kp.x, kp.y);
                par[4] = vp.x;
                par[6] = vp.y;
                const uint32_t there = __ballot_sync(0xffffffffu, now.there);
                const float big = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(vp.x)));  // (never negative)
                if (lane == 0) { s_valid[stage][warp - 8] = there; s_big[stage][warp - 8] = big; }
                fence_proxy_async();
                mbar_arrive(b_full + 8 * stage);
                now = next;
            }
            return true;
        });
    } else if (warp >= 12) {
        // ------------------------------------------------------------ issuing
        regs_down<48>();
        uint32_t n = 0, it = 0;
        if (warp == 12) for_items([&](int, int, int, int, int k0, int k1, bool) {
            bool ok = true;
            if (lane == 0) {
                const uint32_t tiles = smem_u32(s_tiles);
                auto scores = [&](uint32_t m, int x) {     // S of group x for unit m
                    const uint32_t at = tiles + (m & 1) * 2 * TILE + x * 64 * 128;
#pragma unroll
                    for (int s = 0; s < D / 16; ++s)
                        tc_mma(tmem + kS + 64 * x, tmem + kQ + 8 * s, tc_operand(at + (s >> 2) * (kAttUnit * 128) + (s & 3) * 32, 16), tc_shape(64, false), s > 0);
                    tc_commit(b_s + 8 * x);
                };
                ok = wide_wait(b_ready, it & 1, dead) && wide_wait(b_full + 8 * (n & 1), (n >> 1) & 1, dead);
                if (ok) {
                    tc_after_sync();
                    scores(n, 0);
                    scores(n, 1);
                }
                for (int k = k0; ok && k < k1; ++k, ++n) {
                    const uint32_t tile = tiles + ((n & 1) * 2 + 1) * TILE;
                    for (int x = 0; ok && x < 2; ++x) {
                        ok = wide_wait(b_p + 8 * x, n & 1, dead);     // S of this unit is read, P is written
                        if (!ok) break;
                        tc_after_sync();
                        // the next unit's scores first, if its keys are there: the group can go on
                        bool ahead = k + 1 < k1 && mbar_try_wait(b_full + 8 * ((n + 1) & 1), ((n + 1) >> 1) & 1);
                        if (ahead) { tc_after_sync(); scores(n + 1, x); }
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            tc_mma(tmem + kO + D * x, tmem + kP + 32 * x + 8 * s, tc_operand(tile + (x * 64 + s * 16) * 128, kAttUnit * 128), tc_shape(D, true),
                                   k > k0 || s > 0);
                        tc_commit(b_o + 8 * x);
                        if (x == 1) tc_commit(b_empty + 8 * (n & 1));
                        if (k + 1 < k1 && !ahead) {
                            ok = wide_wait(b_full + 8 * ((n + 1) & 1), ((n + 1) >> 1) & 1, dead);
                            if (ok) { tc_after_sync(); scores(n + 1, x); }
                        }
                    }
                }
            }
            n = __shfl_sync(0xffffffffu, n, 0);
            ok = __shfl_sync(0xffffffffu, static_cast<int>(ok), 0);
            ++it;
            return ok;
        });
    } else {
        // ------------------------------------------------------------ softmax
        regs_up<176>();
        const int x = warp >> 2;                    // 0: group A, 1: group B
        const int r = tid & 127;                    // row of the block = lane of tensor memory
        const uint32_t mine = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + mine + kS + 64 * x, t_o = tmem + mine + kO + D * x, t_p = tmem + mine + kP + 32 * x, t_q = tmem + mine + kQ;
        uint32_t n = 0, it = 0;
        for_items([&](int b, int len, int head, int row0, int k0, int k1, bool whole) {
            const int row = row0 + r;
            const bool busy = row0 + (r & ~31) < P.n_rows;        // this warp has rows
            const int prefix = P.prefix_len[b];
            float rho, ra;                          // score in log2 units: ra (scale acc + (mid - 8 scale) rho)
            if (x == 0) {
                // Q to tensor memory, scaled by a power of two to the top of half's range (and to a positive softmax scale)
                const int node = row < P.n_rows ? row / P.group : 0, h = head * P.group + (row - node * P.group);
                const long long at = b * P.q_seq + node * P.q_node + h * P.q_head;
                float most = 0.f, sum = 0.f;
                for (int pass = 0; pass < 2; ++pass) {            // maximum and sum, then the operands
                    int e = most > 0.f ? static_cast<int>(__float_as_uint(most) >> 23) - 126 : 0;
                    e = max(min(e, 112), -110);
                    const float up = __int_as_float((127 + 15 - e) << 23) * (P.scale < 0.f ? -1.f : 1.f);
                    if (pass) {
                        ra = ldexpf(fabsf(P.scale) * 1.4426950408889634f, e - 15 + 24);
                        rho = sum * up * 5.9604644775390625e-8f;  // 2^-24
                    }
#pragma unroll
                    for (int c0 = 0; c0 < D / 32; ++c0) {
                        uint32_t out[16];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {             // eight numbers, one word of codes
                            float v[8];
                            if (row >= P.n_rows) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[i] = 0.f;
                            } else if (P.q_vec) {
                                Elem<DT>::unpack(__ldg(reinterpret_cast<const uint4 *>(static_cast<const char *>(P.q) + 2 * (at + 32 * c0 + 8 * c))), v);
                            } else {
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[i] = load_elem<DT>(P.q, at + 32 * c0 + 8 * c + i);
                            }
                            if (pass == 0) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) { most = fmaxf(most, fabsf(v[i])); sum += v[i]; }
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float f = i & 1 ? up * 0.0625f : up;
                                    out[4 * c + i] = half2_bits(v[i] * f, v[i + 4] * f);
                                }
                            }
                        }
                        __syncwarp();
                        if (pass) tmem_store16(t_q + 16 * c0, out);
                    }
                }
                s_row[0][r] = rho;
                s_row[1][r] = ra;
                for (int i = 0; i * 32 < P.n_nodes; ++i) s_seen[r][i] = 0u;
                for (int a = row < P.n_rows ? node : -1; a >= 0; a = P.parent[a]) s_seen[r][a >> 5] |= 1u << (a & 31);
                __syncwarp();
                tc_wait_st();
                tc_before_sync();
                mbar_arrive(b_ready);
            } else {
                if (!wide_wait_warp(b_ready, it & 1, dead)) return false;
                rho = s_row[0][r];
                ra = s_row[1][r];
            }
            float ref = kNoTop, sum = 0.f, mids = 0.f;
            int expo = -30;                         // ref = maximum + expo, 2^expo at least the largest value scale
            for (int k = k0; k < k1; ++k, ++n) {
                const int stage = n & 1;
                if (!wide_wait_warp(b_full + 8 * stage, (n >> 1) & 1, dead) || !wide_wait_warp(b_s + 8 * x, n & 1, dead)) return false;
                tc_after_sync();
                if (busy) {
                    const float4 *par = s_param + stage * kAttUnit + 64 * x;       // two per pair of keys
                    const int pos0 = k * kAttUnit + 64 * x;
                    const uint32_t ok0 = s_valid[stage][2 * x], ok1 = s_valid[stage][2 * x + 1];
                    const float big = fmaxf(s_big[stage][2 * x], s_big[stage][2 * x + 1]);
                    auto unit = [&](auto plain_tag) {
                        constexpr bool plain = decltype(plain_tag)::value;
                        uint32_t see[2] = {ok0, ok1};             // keys this row sees
                        if (!plain) {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const int first = pos0 + 32 * q - prefix;         // node of bit 0
                                uint32_t m;
                                if (first <= -32) {
                                    m = 0xffffffffu;
                                } else {
                                    // bits first .. first + 31 of the row's nodes, ones below 0
                                    const int wd = first >> 5, sh = first & 31;   // (wd is -1 for a negative first)
                                    const uint32_t lo = wd < 0 ? 0xffffffffu : wd < MCSD_MAX_NODES / 32 && wd * 32 < P.n_nodes ? s_seen[r][wd] : 0u;
                                    const uint32_t hi = (wd + 1) * 32 < P.n_nodes ? s_seen[r][wd + 1] : 0u;
                                    m = __funnelshift_r(lo, hi, sh);
                                }
                                see[q] &= m;
                            }
                        }
                        float2 y[32];
                        float most = -INFINITY;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t acc[16];
                            tmem_load16(t_s + 16 * c, acc);
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const float4 kp = par[2 * (8 * c + j)];
                                const float2 off = __fmul2_rn(make_float2(kp.z, kp.w), make_float2(rho, rho));
                                float2 z = fma2(make_float2(__uint_as_float(acc[2 * j]), __uint_as_float(acc[2 * j + 1])), make_float2(kp.x, kp.y), off);
                                if (!plain) {
                                    if (!((see[c >> 1] >> ((16 * c + 2 * j) & 31)) & 1u)) z.x = -INFINITY;
                                    if (!((see[c >> 1] >> ((16 * c + 2 * j + 1) & 31)) & 1u)) z.y = -INFINITY;
                                }
                                most = max3(most, z.x, z.y);
                                y[8 * c + j] = z;
                            }
                        }
                        // O and P belong to this group once the product of the unit before is done
                        if (n > 0 && !wide_wait_warp(b_o + 8 * x, (n - 1) & 1, dead)) return false;
                        tc_after_sync();
                        const float high = most > -INFINITY ? most * ra : -INFINITY;
                        const bool move = high > ref - static_cast<float>(expo) + kNarrowSlack || (big > 0.f && static_cast<int>(__float_as_uint(big) >> 23) - 126 > expo);
                        if (__any_sync(0xffffffffu, move)) {
                            const float top = ref == kNoTop ? high : fmaxf(ref - static_cast<float>(expo), high);
                            if (big > 0.f) expo = max(expo, static_cast<int>(__float_as_uint(big) >> 23) - 126);
                            const float now = top == -INFINITY ? kNoTop : top + static_cast<float>(expo);
                            const float f = ref == kNoTop ? 0.f : ex2f(ref - now);
                            ref = now;
                            sum *= f;
                            mids *= f;
                            if (k > k0) {
#pragma unroll
                                for (int c = 0; c < D / 16; ++c) {
                                    uint32_t o[16];
                                    tmem_load16(t_o + 16 * c, o);
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                    tmem_store16(t_o + 16 * c, o);
                                }
                            }
                        }
                        float2 s2 = make_float2(0.f, 0.f), m2 = make_float2(0.f, 0.f);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int j = 16 * c + i;
                            const float2 e = fma2(y[j], make_float2(ra, ra), make_float2(-ref, -ref));
                            float2 p = make_float2(ex2f(e.x), ex2f(e.y));
                            float4 vp = par[2 * j + 1];
                            if (!plain) {           // (the parameters of a key that is not seen may be anything)
                                if (!((see[j >> 4] >> ((2 * j) & 31)) & 1u)) { p.x = 0.f; vp.x = vp.z = 0.f; }
                                if (!((see[j >> 4] >> ((2 * j + 1) & 31)) & 1u)) { p.y = 0.f; vp.y = vp.w = 0.f; }
                            }
                            s2 = add2(s2, p);
                            m2 = fma2(p, make_float2(vp.z, vp.w), m2);
                            const float2 q = __fmul2_rn(p, make_float2(vp.x, vp.y));
                            w[i] = half2_bits(q.x, q.y);
                        }
                        tmem_store16(t_p + 16 * c, w);
                        }
                        sum += s2.x + s2.y;
                        mids += m2.x + m2.y;
                        return true;
                    };
                    if ((ok0 & ok1) == 0xffffffffu && pos0 + 64 <= prefix ? !unit(std::true_type()) : !unit(std::false_type())) return false;
                    tc_wait_st();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(b_empty + 8 * stage);  // the parameters are read
                tc_before_sync();
                mbar_arrive(b_p + 8 * x);
            }
            // ---- the end of the item: B hands its rows to A
            if (!wide_wait_warp(b_o + 8 * x, (n - 1) & 1, dead)) return false;
            tc_after_sync();
            if (x == 1) {
                if (it > 0 && !wide_wait_warp(b_free, (it - 1) & 1, dead)) return false;
                if (busy) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_load16(t_o + 16 * c, o);
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            *reinterpret_cast<float4 *>(s_merge + r * (D + 4) + 16 * c + i) =
                                make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
                    }
                    *reinterpret_cast<float4 *>(s_merge + r * (D + 4) + D) = make_float4(ref, sum, mids, 0.f);
                }
                tc_before_sync();
                mbar_arrive(b_merge);
            } else {
                if (!wide_wait_warp(b_merge, it & 1, dead)) return false;
                if (busy) {
                    const float4 other = *reinterpret_cast<const float4 *>(s_merge + r * (D + 4) + D);
                    const float m = fmaxf(ref, other.x);
                    const float fa = att_factor(ref, sum, m), fb = att_factor(other.x, other.y, m);
                    const float l = fmaf(fa, sum, fb * other.y), z = fmaf(fa, mids, fb * other.z);
                    float *part = P.part + static_cast<long long>(2 * blockIdx.x + (k0 > 0 ? 0 : 1)) * part_floats(kWideRows, D);
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        __syncwarp();
                        tmem_load16(t_o + 16 * c, o);
                        if (row < P.n_rows)
#pragma unroll
                        for (int i = 0; i < 16; i += 8) {         // eight columns: one word's codes, in the operands' order
                            float v[8];
#pragma unroll
                            for (int q = 0; q < 8; q += 4) {
                                const float4 ob = *reinterpret_cast<const float4 *>(s_merge + r * (D + 4) + 16 * c + i + q);
                                const float f[4] = {ob.x, ob.y, ob.z, ob.w};
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int p = q + e, d = (p >> 1) + 4 * (p & 1);
                                    v[d] = fmaf(fmaf(fa, __uint_as_float(o[i + p]), fb * f[e]), (p & 2) ? 1048576.f : 16777216.f, z);
                                }
                            }
                            const int at = 16 * c + i;
                            if (whole) {
                                att_store<DT>(P, b, head, row, at, make_float4(v[0], v[1], v[2], v[3]), m, l);
                                att_store<DT>(P, b, head, row, at + 4, make_float4(v[4], v[5], v[6], v[7]), m, l);
                            } else {
                                *reinterpret_cast<float4 *>(part + r * D + at) = make_float4(v[0], v[1], v[2], v[3]);
                                *reinterpret_cast<float4 *>(part + r * D + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
                            }
                        }
                    }
                    if (!whole && row < P.n_rows) { part[kWideRows * D + r] = m; part[kWideRows * (D + 1) + r] = l; }
                }
                __syncwarp();
                tc_before_sync();
                mbar_arrive(b_free);
            }
            ++it;
            return true;
        });
    }
    tc_before_sync();
    __syncthreads();
    if (warp == 12) {
        tc_after_sync();
        tmem_free(tmem, kColumns);
    }
}

}  // namespace mcsd
