// Attention of one new token per sequence over pages that hold rows in 4 bits (quant4.cuh): the first of the two kernels of decode.cu, which
// says what is computed and how the tiles of a layer are shared out; the second one is the same for both.
//
// A token of a unit costs 160 bytes here, 512 there, and the same 4 g d flops: what bounds the kernel is no longer HBM but the instructions that
// make operands of codes, so that these are few and exact:
//   - keys: a code alone in the lower bits of an fp16 is the number c 2^-24 (below the normal ones), one field up 16 c 2^-24, so that a mask makes
//     two operands and one shift per eight codes brings the others down.  Queries are scaled by a power of two per head to where fp16 holds all their bits; which
//     channel is which of the 16 of an instruction is free as long as queries and keys agree.  A group's sum is multiplied by its step afterwards, in fp32.
//   - values: their step differs from token to token, over which the instruction sums, so it has to be in the operand.  A code in the lower bits of a
//     bf16 is c 2^-133, one field up 16 c 2^-133 (which runs on into the first normal numbers); two products, with 2^126 and with 2^7 s or 2^3 s,
//     make s c of it (s has four significant bits, so that this is exact).  The pairs are tokens: a permutation per two words brings the
//     same channels of two tokens side by side.
//   - lo enters once for a group, not for every channel.  q.k = sum_c q_c s c + sum_groups lo_g (sum of the group's q): one more
//     matrix instruction per tile with the least values as rows and the sums of the query, in three bf16 terms (24 bits), as columns.
//     sum_j p_j v_j likewise gets one more instruction, whose sums are added to the channels at the end.
//   - values are summed as s (c - 7) and lo + 7 s, not as s c and lo: of values on both sides of 0 the latter are two sums of one sign each, over a long
//     context some hundred times their own sum, and fp32 rounds them accordingly (16 heads x 131072 tokens: 28 % of the outputs were not the bf16 nearest to the
//     exact ones, now 0.4 %, for 51.0 -> 53.3 us of 8 heads, g = 5).  7 and not 7.5 because steps are rounded up, which takes the middle code down.  s (c - 7) is
//     exact in bf16 and free, as the product with s has a summand; lo + 7 s is two bf16 terms, exact as well, in the two halves of the instruction's rows.
// So every product that a matrix instruction sees is exact but for the weights' two bf16 terms, as in the other kernel, and for query channels some 2^-27 below
// their head's greatest (query_operands).
//
// The rows of a page lie back to back, so that a tile of 16 is 1280 bytes in one piece (two on pages of 8): five 16-byte copies per lane for
// K and V together.  Twelve warps of 168 registers take two tiles a step, which the compiler interleaves; beyond eight heads eight warps of 255 (nothing is spilled).
//
// Measured (both kernels, one layer, device time of calls in a row): 8 heads x 131072 tokens 49.4 - 50.2 us for 1 to 8 query heads (bf16: 89), 75 for 12,
// 76 for 16, 133 for 32, 252 for 64; with weights 57 - 58.5; capped 54.  16 ragged sequences x 8 heads, 470 K tokens, with weights, 41.  The copies alone take 34,
// the arithmetic alone 47 (before values were summed about their middle, the whole 47.3).  437 instructions per tile of 16 tokens (712 at first), 61 % of the issue
// slots, the logic pipe 39 %, the tensor pipe 20 %; the largest stall is the latency of dependent instructions, at three warps a scheduler.  A matrix instruction also
// holds up the others for three of its nine cycles.  Not better (before that as well): 16 warps of 128 registers (57 us), 8 of 255 (59); scores of a tile beside the product
// of the one before (57); codes as e4m3 for the instruction of 8-bit types, which is made of fp16 ones here (68); both terms of the weights in the
// eight columns of one instruction for up to four heads (2 us less for long contexts, nothing else).
#include "decode.cuh"
#include "quant4.cuh"

#include <cuda_fp16.h>

#include <type_traits>

namespace compactor {
namespace {

using namespace decode;

constexpr int kTileBytes = kTile * kRow4;              // of K, or of V
constexpr int kStageBytes = 2 * kTileBytes;

template <int NG> struct Four {
    static constexpr int kWarps = NG == 1 ? kDecode4Warps : kDecode4WarpsWide;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kStages = NG == 1 ? 5 : 8;    // 154 KB, 164 KB
    static constexpr size_t kSmemBytes = (size_t)kWarps * kStages * kStageBytes;
};

// The 32 channels that a lane multiplies: 32 g + 8 tig + 0..7, of head t * 8 + gid.
template <int NG>
__device__ __forceinline__ void load_queries(const DecodeArgs& a, const Cursor& c, uint4 (&q)[NG][4], int lane) {
    const int gid = lane >> 2, tig = lane & 3;
    const int h = c.unit / a.c.batch, b = c.unit - h * a.c.batch;
    const int head0 = h * a.g + c.grp * kDecodeHeads, heads = min(kDecodeHeads, a.g - c.grp * kDecodeHeads);
#pragma unroll
    for (int t = 0; t < NG; ++t) {
        const bool on = t * 8 + gid < heads;
        const uint4* src = reinterpret_cast<const uint4*>(a.q + b * a.q_seq + (long long)(head0 + (on ? t * 8 + gid : 0)) * a.q_head);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            q[t][g] = src[4 * g + tig];
            if (!on) q[t][g] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// B operands of a unit's queries: of the lane's eight channels of group g the pairs (0, 4) and (2, 6), then (1, 5) and (3, 7) times 2^-4, as
// fp16 of q 2^k; the sums of a group's channels, group tig, times 2^(k - 24), as three bf16 terms; and for the two heads of the lane's scores
// 2^(24 - k).  k brings the head's greatest channel to 2^14 .. 2^15.  The last place of an fp16 is never below 2^-24, so that the eight bits of a bf16 are all held
// down to 2^-31 of that channel's power of two, those of odd channels, because of the 2^-4, to 2^-27; below, a channel is off by at most 2^-39, or
// 2^-35, of it.  Queries of 2^118 and more, whose scale back to a score would be beyond fp32, and those that are not finite make all of their head's scores
// not a number (as infinite ones, the scores of a head could all be -inf, and its row zero).
template <int NG>
__device__ __forceinline__ void query_operands(const uint4 (&q)[NG][4], uint32_t (&qf)[NG][4][2][2], uint32_t (&qs)[NG][2], float (&unscale)[NG][2], int lane) {
    const int tig = lane & 3;
#pragma unroll
    for (int t = 0; t < NG; ++t) {
        uint32_t top = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint4 x = q[t][g];
            top = max_nan2(top, max_nan2(max_nan2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), max_nan2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
        }
        top = max_nan2(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max_nan2(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = max_nan2(top, top >> 16 | top << 16);
        const int k = max(-102, min(141 - (int)((top >> 7) & 255u), 126));
        const float up = __int_as_float((k + 127) << 23), down = __int_as_float((127 + 24 - k) << 23);
        float mine = 0.f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint4 x = q[t][g];
            float sum = 0.f;
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                const uint32_t w[4] = {x.x, x.z, x.y, x.w};
                const float by = odd == 0 ? up : up * 0.0625f;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float lo = odd == 0 ? bf16_lo(w[2 * i]) : bf16_hi(w[2 * i]), hi = odd == 0 ? bf16_lo(w[2 * i + 1]) : bf16_hi(w[2 * i + 1]);
                    sum += lo + hi;
                    const __half2 h = __floats2half2_rn(lo * by, hi * by);
                    qf[t][g][odd][i] = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if (g == tig) mine = sum;
        }
        mine = (top & 0x7fffu) >= 0x7a80u ? __int_as_float(0x7fffffff) : mine * (up * 0x1p-24f);      // (the bits of 2^118)
        const float t0 = __bfloat162float(__float2bfloat16_rn(mine)), r0 = mine - t0;
        const float t1 = __bfloat162float(__float2bfloat16_rn(r0)), t2 = r0 - t1;
        qs[t][0] = pack_bf16(t0, t1);
        qs[t][1] = pack_bf16(t2, 0.f);
        unscale[t][0] = __shfl_sync(0xffffffffu, down, 8 * tig);
        unscale[t][1] = __shfl_sync(0xffffffffu, down, 8 * tig + 4);
    }
}

constexpr uint32_t kFirst = 0x000f000fu, kSecond = 0x00f000f0u;      // codes of two channels as they are: in fp16 c 2^-24 and c 2^-20, in bf16 c 2^-133 and c 2^-129

// The instruction of decode.cuh, free to be placed where its operands are ready.
__device__ __forceinline__ void mma4(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// lo + 7 s of two tokens as two terms whose sum is exact: what a sum of two bf16 is rounded by is a bf16 itself.  less: -7 s.
__device__ __forceinline__ void middle(uint32_t lo, uint32_t less, uint32_t& sum, uint32_t& rest) {
    sum = sub2(lo, less);
    const uint32_t of_s = sub2(sum, lo), of_lo = sub2(sum, of_s);        // the shares of 7 s and of lo in the rounded sum
    rest = sub2(sub2(lo, of_lo), add2(of_s, less));
}

// The same in fp16: codes of keys times queries.
__device__ __forceinline__ void mma_codes(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// CAP: scores are capped.  ACC: weights are accumulated.
template <int NG, bool CAP, bool ACC>
__global__ void __launch_bounds__(Four<NG>::kThreads, 1)
decode4_kernel(const __grid_constant__ DecodeArgs a) {
    constexpr int kWarps = Four<NG>::kWarps, kThreads = Four<NG>::kThreads, kStages = Four<NG>::kStages;
    extern __shared__ __align__(1024) unsigned char ring[];
    __shared__ int cum[kThreads + 1];
    __shared__ int warp_sum[kWarps];
    __shared__ int new_page[kWarps][kStages];
    __shared__ int live[kUnitsInSmem];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    pdl_wait();

    // cost before each thread's run of units
    const int per = (a.units + kThreads - 1) / kThreads;
    const int u0 = min(a.units, tid * per), u1 = min(a.units, u0 + per);
    int mine = 0;
    for (int u = u0; u < u1; ++u) {
        const int n = live_tokens(a, u);
        if (u < kUnitsInSmem) live[u] = n;
        mine += cost_of(n);
    }
    int incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) before += w < warp ? warp_sum[w] : 0;
    cum[tid + 1] = before + incl;
    if (tid == 0) cum[0] = 0;
    __syncthreads();
    const int all = cum[kThreads];
    if (blockIdx.x == 0) {                                   // for the second kernel, and the units that are refused
        int at = cum[tid];
        for (int u = u0; u < u1; ++u) {
            a.prefix[u] = at;
            at += cost_of(live_tokens(a, u));
            const int n = __ldcg(a.lengths + u);
            if (a.status != nullptr && n >= 0 && (long long)n + (a.k_new != nullptr) > a.capacity)
                atomicOr(a.status + u, COMPACTOR_STATUS_CAPACITY);
        }
        if (tid == 0) a.prefix[a.units] = all;
    }
    const int total = all * a.groups;
    const int workers = active_workers(a, total);
    const int worker = warp * gridDim.x + blockIdx.x;        // neighbouring workers on different SMs: a small call uses them all
    if (worker >= workers) return;
    const Share share(total, workers);
    const int begin = share.begin(worker);
    int left_p = share.size(worker);                         // cost that the producer has not passed yet

    // the unit that holds place `begin`
    Cursor start;
    {
        int lo = 0, hi = kThreads;                           // cum[lo] * groups <= begin < cum[hi] * groups
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cum[mid] * a.groups <= begin) lo = mid; else hi = mid;
        }
        int left = begin - cum[lo] * a.groups;
        auto tokens_of = [&](int unit) { return unit < kUnitsInSmem ? live[unit] : live_tokens(a, unit); };
        int u = lo * per, n = tokens_of(u);
        while (left >= cost_of(n) * a.groups) {
            left -= cost_of(n) * a.groups;
            n = tokens_of(++u);
        }
        start.unit = u; start.tokens = n; start.tiles = tiles_of(n);
        start.grp = left / cost_of(n);
        start.tile = left - start.grp * cost_of(n) - kUnitCost;
        if (start.tile < 0) {                                // within the unit's head: the first tile is the next
            left_p += start.tile;
            start.tile = 0;
            if (left_p <= 0) return;
        }
    }
    int left_c = left_p;                                     // cost that the consumer has not passed yet

    unsigned char* my_ring = ring + (size_t)warp * kStages * kStageBytes;
    const uint32_t ring_s = smem_u32(my_ring);

    // ---- producer: one tile into a stage.  Lane l copies the 16-byte pieces l, l + 32 and l + 64 of the 80 of either tile; pieces 0 .. 39 are rows 0 .. 7.
    // A tile that goes on in the page of the one before it (run > 0) is where that one ended; else its page ids are looked up.  They are asked
    // for ahead as in the other kernel: 64 page ids of the unit (lane l holds entries e0 + l and e0 + 32 + l) and the first 32 of the unit after it.
    // (The queries are not, but for the first unit's: the registers that would hold them are worth more than the wait.)
    Cursor pc = start, nc = start;
    int e0 = (pc.tile * kTile) >> a.c.page_shift;
    int ids = page_ids(a, pc, e0, lane), ids_after = page_ids(a, pc, e0 + 32, lane), ids_next_unit = -1;
    uint4 q_first[NG][4];
    load_queries<NG>(a, pc, q_first, lane);
    if (nc.next_unit(a, live)) ids_next_unit = page_ids(a, nc, 0, lane);
    const int appended = a.k_new != nullptr ? 1 : 0;
    const long long v_from_k = reinterpret_cast<const char*>(a.c.v) - reinterpret_cast<const char*>(a.c.k);
    const char* src = nullptr;                               // where the next tile of the page begins, for this lane
    int run = 0;                                             // tiles left in the page
    int full = (pc.tokens - appended) / kTile;               // tiles of the unit whose rows are all in pages
    uint32_t bad = 0;                                        // two bits per stage: a half of its tile is on a page that is none
    int in_stage = 0;
    auto issue = [&]() {
        if (left_p > 0) {
            const uint32_t ks = ring_s + in_stage * kStageBytes + lane * 16;
            bad &= ~(3u << (2 * in_stage));
            bool whole = pc.tile < full;
            const int base = pc.tile * kTile, e = base >> a.c.page_shift;
            int p0 = -1;
            if (run > 0 && whole) {
                --run;
                p0 = 0;
            } else if (whole && a.c.page_shift >= 4) {       // one page: little to look up, which on pages of 16 is for every tile (8 heads x 131072 51.1 -> 50.3 us, now 52.5; ragged 71.4 -> 69.7)
                if (e >= e0 + 32) {
                    e0 += 32;
                    ids = ids_after;
                    ids_after = page_ids(a, pc, e0 + 32, lane);
                }
                p0 = __shfl_sync(0xffffffffu, ids, e - e0);
                if ((unsigned)p0 >= (unsigned)a.c.n_pages) p0 = -1;
                src = reinterpret_cast<const char*>(a.c.k + row_in_pool(a.c, max(p0, 0), base)) + lane * 16;
                run = ((1 << a.c.page_shift) - (base & ((1 << a.c.page_shift) - 1))) / kTile - 1;
            }
            if (p0 < 0) {                                    // two pages of 8, or rows that are in no page or behind the last token: zeros
                run = 0;
                whole = false;
                const int n = pc.tokens, cached = n - appended;
                if (e + 1 >= e0 + 32) {                      // (pages of 8 tokens: a tile has two)
                    e0 += 32;
                    if (e < e0) {                            // a tile on the seam keeps one entry of the old run
                        const int seam = __shfl_sync(0xffffffffu, ids, 31);
                        const int rest = __shfl_up_sync(0xffffffffu, ids_after, 1);
                        ids = lane == 0 ? seam : rest;
                        e0 -= 1;
                        ids_after = page_ids(a, pc, e0 + 32, lane);
                    } else {
                        ids = ids_after;
                        ids_after = page_ids(a, pc, e0 + 32, lane);
                    }
                }
                p0 = __shfl_sync(0xffffffffu, ids, e - e0);
                int p1 = __shfl_sync(0xffffffffu, ids, ((base + 8) >> a.c.page_shift) - e0);
                if ((unsigned)p0 >= (unsigned)a.c.n_pages) p0 = -1;
                if ((unsigned)p1 >= (unsigned)a.c.n_pages || base + 8 >= n) p1 = -1;
                src = reinterpret_cast<const char*>(a.c.k + row_in_pool(a.c, max(p0, 0), base)) + lane * 16;
                // pieces of the second half, as if its run of 640 bytes had begun before it
                const char* src1 = reinterpret_cast<const char*>(a.c.k + row_in_pool(a.c, max(p1, 0), base + 8)) + lane * 16 - 8 * kRow4;
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const int at = lane + 32 * i, tok = base + at / 5;
                    if (at >= kTileBytes / 16) continue;
                    const bool on = tok < cached && (at < 40 ? p0 : p1) >= 0;
                    const char* from = on ? (at < 40 ? src : src1) + 512 * i : reinterpret_cast<const char*>(a.c.k);
                    cp_async16(ks + 512 * i, from, on ? 16 : 0);
                    cp_async16(ks + kTileBytes + 512 * i, from + v_from_k, on ? 16 : 0);
                }
                const int fresh_row = cached < n ? cached - base : -1;   // the new token's row of this tile, if it has it
                const uint32_t bits = (p0 < 0 && base < cached ? 1u : 0u) | (p1 < 0 && base + 8 < cached ? 2u : 0u);
                const int np = fresh_row < 8 ? p0 : p1;
                bad |= bits << (2 * in_stage);
                if (lane == 0) {
                    new_page[warp][in_stage] = np;
                    if (a.status != nullptr && (bits != 0 || (fresh_row >= 0 && fresh_row < kTile && np < 0)))
                        atomicOr(a.status + pc.unit, COMPACTOR_STATUS_PAGE);
                }
            }
            if (whole) {
                const char* sv = src + v_from_k;
                cp_async16(ks, src);
                cp_async16(ks + kTileBytes, sv);
                cp_async16(ks + 512, src + 512);
                cp_async16(ks + kTileBytes + 512, sv + 512);
                if (lane < 16) {
                    cp_async16(ks + 1024, src + 1024);
                    cp_async16(ks + kTileBytes + 1024, sv + 1024);
                }
                src += kTileBytes;
            }
            in_stage = in_stage + 1 == kStages ? 0 : in_stage + 1;
            --left_p;
            if (++pc.tile == pc.tiles && (left_p -= kUnitCost) > 0) {
                pc = nc;
                e0 = 0;
                run = 0;
                full = (pc.tokens - appended) / kTile;
                ids = ids_next_unit;
                ids_after = page_ids(a, pc, 32, lane);
                if (nc.next_unit(a, live)) ids_next_unit = page_ids(a, nc, 0, lane);
            }
        }
        cp_commit();
    };
#pragma unroll 1
    for (int s = 0; s < kStages; ++s) issue();

    // ---- consumer
    // The exponentials are taken against a reference that follows a head's maximum only when a score is more than 2^kSlack above it, so that most
    // tiles need neither the maximum over the warp's lanes nor a new scale of what is summed.
    constexpr float kSlack = 8.f;
    Cursor cc = start;
    const float scale2 = CAP ? a.scale / a.softcap : a.scale * kLog2e, cap_out = CAP ? a.softcap * kLog2e : 0.f;
    uint32_t qf[NG][4][2][2], qs[NG][2];
    float to_base2[NG][2];                                   // from the scores as they are summed (when they are capped, to what the cap takes)
    float o[NG][8][4], ol[NG][4];
    float ref[NG][2], most[NG][2], sum[NG][2];               // reference in base 2; score above which it has to follow (-inf: none yet)
    int first_tile = 0, head0 = 0, heads = 0, stage = 0;
    auto enter = [&](const uint4 (&q)[NG][4]) {              // a new unit or group
        first_tile = cc.tile;
        head0 = cc.unit / a.c.batch * a.g + cc.grp * kDecodeHeads;
        heads = min(kDecodeHeads, a.g - cc.grp * kDecodeHeads);
        query_operands<NG>(q, qf, qs, to_base2, lane);
#pragma unroll
        for (int t = 0; t < NG; ++t) {
#pragma unroll
            for (int s = 0; s < 8; ++s) o[t][s][0] = o[t][s][1] = o[t][s][2] = o[t][s][3] = 0.f;
            ol[t][0] = ol[t][1] = ol[t][2] = ol[t][3] = 0.f;
#pragma unroll
            for (int c = 0; c < 2; ++c)
                // (Queries times a scale beyond 2^117 end at 2^127 and have their scores too small by the rest: among keys above 2^-110 they are still
                // so far apart that one token takes all.)
                to_base2[t][c] = fminf(fmaxf(to_base2[t][c] * scale2, 0x1p-149f), 0x1p127f);     // (never 0 or infinite: -inf stays -inf, 0 stays 0)
            ref[t][0] = ref[t][1] = 0.f;
            most[t][0] = most[t][1] = -INFINITY;
            sum[t][0] = sum[t][1] = 0.f;
        }
    };
    enter(q_first);

    while (true) {
        if (left_c <= kStages) pdl_trigger();                // the second kernel's blocks are let in when the tiles run out
        const int cached = cc.tokens - appended;
        // COUNT tiles of the unit, whose steps the compiler interleaves
        auto attend = [&](auto count) {
            constexpr int COUNT = decltype(count)::value;
            cp_wait<kStages - COUNT>();
            __syncwarp();
            unsigned char* tile[COUNT];
            int base[COUNT];
            uint32_t bits[COUNT];
            bool ragged = false;                             // some rows are not the cache's
#pragma unroll
            for (int u = 0; u < COUNT; ++u) {
                const int at = stage + u < kStages ? stage + u : stage + u - kStages;
                tile[u] = my_ring + at * kStageBytes;
                base[u] = (cc.tile + u) * kTile;
                bits[u] = (bad >> (2 * at)) & 3u;
                ragged |= base[u] + kTile > cached || bits[u] != 0;
            }
            if (ragged && cached < cc.tokens && cached < base[COUNT - 1] + kTile && cached >= base[0]) {
                // the new token's rows: held in 4 bits first, in the tile and, by the first group, in its page; lanes 0 .. 15 have K's, the others V's
                const int which = COUNT > 1 && cached >= base[COUNT - 1] ? COUNT - 1 : 0;
                const int at_stage = stage + which < kStages ? stage + which : stage + which - kStages;
                const int h = cc.unit / a.c.batch, b = cc.unit - h * a.c.batch, piece = lane & 15;
                const __nv_bfloat16* from = lane < 16 ? a.k_new + b * a.kn_seq + h * a.kn_head : a.v_new + b * a.vn_seq + h * a.vn_head;
                uint32_t param;
                const uint32_t codes = quantise8(*(reinterpret_cast<const uint4*>(from) + piece), param);
                unsigned char* row = my_ring + at_stage * kStageBytes + (lane < 16 ? 0 : kTileBytes) + (cached & (kTile - 1)) * kRow4;
                *reinterpret_cast<uint32_t*>(row + 4 * piece) = codes;
                if ((piece & 3) == 0) *reinterpret_cast<uint32_t*>(row + kRow4Codes + piece) = param;
                const int page = new_page[warp][at_stage];
                if (page >= 0 && cc.grp == 0) {
                    row = reinterpret_cast<unsigned char*>((lane < 16 ? a.c.k : a.c.v) + row_in_pool(a.c, page, cached));
                    *reinterpret_cast<uint32_t*>(row + 4 * piece) = codes;
                    if ((piece & 3) == 0) *reinterpret_cast<uint32_t*>(row + kRow4Codes + piece) = param;
                    const long long at = slot_in_pool(a.c, page, cached);
                    if (lane == 0 && a.c.positions != nullptr)
                        a.c.positions[at] = a.new_positions != nullptr ? a.new_positions[cc.unit % a.c.batch] : cached;
                    if (lane == 0 && a.c.mass != nullptr && !ACC) a.c.mass[at] = 0.f;
                }
                __syncwarp();
            }

            // S^T: 16 tokens x 8 NG heads
            float s[COUNT][NG][4];
#pragma unroll
            for (int u = 0; u < COUNT; ++u) {
#pragma unroll
                for (int t = 0; t < NG; ++t) s[u][t][0] = s[u][t][1] = s[u][t][2] = s[u][t][3] = 0.f;
                const unsigned char* ra = tile[u] + gid * kRow4;
                const unsigned char* rb = ra + 8 * kRow4;
                const uint32_t la = *reinterpret_cast<const uint32_t*>(ra + kRow4Codes + 4 * tig), lb = *reinterpret_cast<const uint32_t*>(rb + kRow4Codes + 4 * tig);
                const uint32_t la2 = __byte_perm(la, 0u, 0x3232), lb2 = __byte_perm(lb, 0u, 0x3232);
                const uint32_t lf[4] = {la2, lb2, la2, lb2};
#pragma unroll
                for (int t = 0; t < NG; ++t) mma4(s[u][t], lf, qs[t][0], qs[t][1]);
                const uint4 pa = *reinterpret_cast<const uint4*>(ra + kRow4Codes), pb = *reinterpret_cast<const uint4*>(rb + kRow4Codes);
                const uint32_t para[4] = {pa.x, pa.y, pa.z, pa.w}, parb[4] = {pb.x, pb.y, pb.z, pb.w};
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t wa = *reinterpret_cast<const uint32_t*>(ra + 16 * g + 4 * tig), wb = *reinterpret_cast<const uint32_t*>(rb + 16 * g + 4 * tig);
                    const uint32_t wa8 = wa >> 8, wb8 = wb >> 8;
                    const uint32_t kf[2][4] = {{wa & kFirst, wb & kFirst, wa8 & kFirst, wb8 & kFirst}, {wa & kSecond, wb & kSecond, wa8 & kSecond, wb8 & kSecond}};
                    const float sa = bf16_lo(para[g]), sb = bf16_lo(parb[g]);
#pragma unroll
                    for (int t = 0; t < NG; ++t) {
                        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int odd = 0; odd < 2; ++odd) mma_codes(x, kf[odd], qf[t][g][odd][0], qf[t][g][odd][1]);
                        s[u][t][0] = fmaf(sa, x[0], s[u][t][0]); s[u][t][1] = fmaf(sa, x[1], s[u][t][1]);
                        s[u][t][2] = fmaf(sb, x[2], s[u][t][2]); s[u][t][3] = fmaf(sb, x[3], s[u][t][3]);
                    }
                }
            }
            if (CAP) {
#pragma unroll
                for (int u = 0; u < COUNT; ++u)
#pragma unroll
                    for (int t = 0; t < NG; ++t)
#pragma unroll
                        for (int c = 0; c < 4; ++c) s[u][t][c] = cap_out * tanhf(s[u][t][c] * to_base2[t][c & 1]);
            }
            if (ragged) {                                    // what does not count gets -inf
#pragma unroll
                for (int u = 0; u < COUNT; ++u) {
                    const int ta = base[u] + gid, tb = ta + 8;
                    const bool la = ta < cc.tokens && !((bits[u] & 1) && ta < cached), lb = tb < cc.tokens && !((bits[u] & 2) && tb < cached);
#pragma unroll
                    for (int t = 0; t < NG; ++t) {
                        if (!la) s[u][t][0] = s[u][t][1] = -INFINITY;
                        if (!lb) s[u][t][2] = s[u][t][3] = -INFINITY;
                    }
                }
            }
            if (ACC) {                                       // kept, in base 2, until the sum over the whole unit is known
                float* col = a.scores + ((long long)cc.unit * a.g + cc.grp * kDecodeHeads + 2 * tig) * a.unit_rows + base[0] + gid;
#pragma unroll
                for (int t = 0; t < NG; ++t)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        if (t * 8 + 2 * tig + c < heads) {   // 32 bytes of a head's scores per group of eight lanes
                            float* at = col + (long long)(t * 8 + c) * a.unit_rows;
#pragma unroll
                            for (int u = 0; u < COUNT; ++u) {
                                at[kTile * u] = s[u][t][c] * (CAP ? 1.f : to_base2[t][c]);
                                at[kTile * u + 8] = s[u][t][c + 2] * (CAP ? 1.f : to_base2[t][c]);
                            }
                        }
            }
            bool above = false;
#pragma unroll
            for (int u = 0; u < COUNT; ++u)
#pragma unroll
                for (int t = 0; t < NG; ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) above |= s[u][t][c] > most[t][c & 1];
            if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                for (int t = 0; t < NG; ++t) {
                    float by[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = fmaxf(s[0][t][c], s[0][t][c + 2]);
#pragma unroll
                        for (int u = 1; u < COUNT; ++u) m = fmaxf(m, fmaxf(s[u][t][c], s[u][t][c + 2]));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)) * (CAP ? 1.f : to_base2[t][c]);
                        const bool none = most[t][c] == -INFINITY;           // nothing summed yet
                        const float now = m == -INFINITY ? ref[t][c] : none ? m : fmaxf(m, ref[t][c]);
                        by[c] = none ? 1.f : ex2f(ref[t][c] - now);
                        ref[t][c] = now;
                        sum[t][c] *= by[c];
                        if (m != -INFINITY) most[t][c] = CAP ? now + kSlack : (now + kSlack) / to_base2[t][c];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        o[t][j][0] *= by[0]; o[t][j][1] *= by[1];
                        o[t][j][2] *= by[0]; o[t][j][3] *= by[1];
                    }
                    ol[t][0] *= by[0]; ol[t][1] *= by[1];
                    ol[t][2] *= by[0]; ol[t][3] *= by[1];
                }
            }
            uint32_t pf[COUNT][NG][2], pl[COUNT][NG][2];     // weights as two bf16 terms, the first cut off, the second rounded: within 2^-16
#pragma unroll
            for (int u = 0; u < COUNT; ++u)
#pragma unroll
                for (int t = 0; t < NG; ++t)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // (the product is rounded as the reference's was: scores of 2^31 and more, whose last place is a whole power, are told apart by that)
                        const float x = ex2f(CAP ? s[u][t][2 * i] - ref[t][0] : __fadd_rn(__fmul_rn(s[u][t][2 * i], to_base2[t][0]), -ref[t][0]));
                        const float y = ex2f(CAP ? s[u][t][2 * i + 1] - ref[t][1] : __fadd_rn(__fmul_rn(s[u][t][2 * i + 1], to_base2[t][1]), -ref[t][1]));
                        sum[t][0] += x; sum[t][1] += y;
                        const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
                        pf[u][t][i] = transpose8x8(__byte_perm(xb, yb, 0x7632));
                        pl[u][t][i] = transpose8x8(pack_bf16(x - __uint_as_float(xb & 0xffff0000u), y - __uint_as_float(yb & 0xffff0000u)));
                    }
            // O^T += V^T P^T: 128 channels x 8 NG heads.  The lane has the 16 channels 16 gid + 0..15 of tokens 2 tig, + 1, + 8 and + 9; row gid of the
            // j-th instruction is channel 16 gid + j, row gid + 8 is 16 gid + 8 + j.
#pragma unroll
            for (int u = 0; u < COUNT; ++u) {
                const unsigned char* r = tile[u] + kTileBytes + 2 * tig * kRow4;
                uint2 v[4];
                uint32_t par[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned char* row = r + ((i & 1) + (i >> 1) * 8) * kRow4;
                    v[i] = *reinterpret_cast<const uint2*>(row + 8 * gid);
                    par[i] = *reinterpret_cast<const uint32_t*>(row + kRow4Codes + 4 * (gid >> 1));
                }
                const uint32_t s0 = __byte_perm(par[0], par[1], 0x5410), s1 = __byte_perm(par[2], par[3], 0x5410);
                const uint32_t s0f = fma2(s0, 0x43004300u, 0u), s1f = fma2(s1, 0x43004300u, 0u), s0s = fma2(s0, 0x41004100u, 0u), s1s = fma2(s1, 0x41004100u, 0u);
                const uint32_t s0m = fma2(s0, 0xc0e0c0e0u, 0u), s1m = fma2(s1, 0xc0e0c0e0u, 0u);         // -7 s
#pragma unroll
                for (int j4 = 0; j4 < 8; j4 += 4) {          // the same four channels of two tokens in the halves of a word
                    const unsigned sel = j4 == 0 ? 0x5410 : 0x7632;
                    const uint32_t x[4] = {__byte_perm(v[0].x, v[1].x, sel), __byte_perm(v[0].y, v[1].y, sel), __byte_perm(v[2].x, v[3].x, sel), __byte_perm(v[2].y, v[3].y, sel)};
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const int j = j4 + n;
                        uint32_t vf[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t c = (n < 2 ? x[i] : x[i] >> 8) & ((n & 1) == 0 ? kFirst : kSecond);
                            vf[i] = fma2(fma2(c, 0x7e807e80u, 0u), (n & 1) == 0 ? (i < 2 ? s0f : s1f) : (i < 2 ? s0s : s1s), i < 2 ? s0m : s1m);
                        }
#pragma unroll
                        for (int t = 0; t < NG; ++t) mma4(o[t][j], vf, pf[u][t][0], pf[u][t][1]);
#pragma unroll
                        for (int t = 0; t < NG; ++t) mma4(o[t][j], vf, pl[u][t][0], pl[u][t][1]);
                    }
                }
                uint32_t lf[4];
                middle(__byte_perm(par[0], par[1], 0x7632), s0m, lf[0], lf[1]);
                middle(__byte_perm(par[2], par[3], 0x7632), s1m, lf[2], lf[3]);
#pragma unroll
                for (int t = 0; t < NG; ++t) mma4(ol[t], lf, pf[u][t][0], pf[u][t][1]);
#pragma unroll
                for (int t = 0; t < NG; ++t) mma4(ol[t], lf, pl[u][t][0], pl[u][t][1]);
            }
            __syncwarp();
#pragma unroll 1
            for (int u = 0; u < COUNT; ++u) issue();
            stage += COUNT;
            if (stage >= kStages) stage -= kStages;
            left_c -= COUNT;
            cc.tile += COUNT;
        };
        if (left_c >= 2 && cc.tile + 1 < cc.tiles) attend(std::integral_constant<int, 2>());
        else attend(std::integral_constant<int, 1>());

        const bool unit_ends = cc.tile == cc.tiles;
        if (unit_ends) left_c -= kUnitCost;
        if (unit_ends || left_c <= 0) {                      // hand over what this warp has of the unit
            const long long slot = (long long)worker + cc.unit * a.groups + cc.grp;
            const bool whole = unit_ends && first_tile == 0;
            const int b = cc.unit % a.c.batch, gg = min(a.g, kDecodeHeads);
#pragma unroll
            for (int t = 0; t < NG; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float l = sum[t][c];
                    l += __shfl_xor_sync(0xffffffffu, l, 4);
                    l += __shfl_xor_sync(0xffffffffu, l, 8);
                    l += __shfl_xor_sync(0xffffffffu, l, 16);
                    const int head = t * 8 + 2 * tig + c;
                    if (head >= heads) continue;
                    if (gid == 0) {
                        a.ml[slot * 32 + head] = most[t][c] == -INFINITY ? -INFINITY : ref[t][c];
                        a.ml[slot * 32 + 16 + head] = l;
                    }
                    float x[16];
#pragma unroll
                    for (int j = 0; j < 8; ++j) { x[j] = (o[t][j][c] + ol[t][c]) + ol[t][c + 2]; x[8 + j] = (o[t][j][c + 2] + ol[t][c]) + ol[t][c + 2]; }
                    if (whole) {
                        const float inv = l == 0.f ? 0.f : 1.f / l;
                        uint4* dst = reinterpret_cast<uint4*>(a.out + b * a.out_seq + (long long)(head0 + head) * a.out_head + 16 * gid);
#pragma unroll
                        for (int i = 0; i < 16; i += 8)
                            dst[i / 8] = make_uint4(pack_bf16(x[i] * inv, x[i + 1] * inv), pack_bf16(x[i + 2] * inv, x[i + 3] * inv),
                                                    pack_bf16(x[i + 4] * inv, x[i + 5] * inv), pack_bf16(x[i + 6] * inv, x[i + 7] * inv));
                        if (gid == 0 && a.lse != nullptr)
                            a.lse[(long long)b * (a.c.heads * a.g) + head0 + head] = l == 0.f ? -INFINITY : kLn2 * (ref[t][c] + log2f(l));
                    } else {
                        float4* dst = reinterpret_cast<float4*>(a.o + (slot * gg + head) * kD + 16 * gid);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    }
                }
            if (left_c <= 0) return;
            cc.next_unit(a, live);
            uint4 q[NG][4];
            load_queries<NG>(a, cc, q, lane);
            enter(q);
        }
    }
}

}  // namespace

namespace {
template <int NG, bool CAP, bool ACC>
cudaError_t launch(const DecodeArgs& a, cudaStream_t stream) {
    static std::atomic<unsigned long long> done;
    const cudaError_t e = allow_smem(decode4_kernel<NG, CAP, ACC>, (int)Four<NG>::kSmemBytes, done);
    if (e != cudaSuccess) return e;
    return launch_chained(kPdlOther, decode4_kernel<NG, CAP, ACC>, dim3(a.workers / Four<NG>::kWarps), dim3(Four<NG>::kThreads), Four<NG>::kSmemBytes, stream, a);
}
template <int NG>
cudaError_t launch(const DecodeArgs& a, cudaStream_t stream) {
    if (a.softcap > 0.f) return a.accumulate ? launch<NG, true, true>(a, stream) : launch<NG, true, false>(a, stream);
    return a.accumulate ? launch<NG, false, true>(a, stream) : launch<NG, false, false>(a, stream);
}
}  // namespace

cudaError_t launch_decode4(const DecodeArgs& a, cudaStream_t stream) { return a.g <= 8 ? launch<1>(a, stream) : launch<2>(a, stream); }

}  // namespace compactor
