// Attention of one new token per sequence over a paged cache whose every (KV head, sequence) unit has its own pages
// and its own length:
//
//   y_j = scale q.k_j   (or c tanh(scale q.k_j / c)),   p = softmax(y),   o = sum_j p_j v_j,   lse = log sum_j e^{y_j},
//
// for the g query heads of each KV head, with the new token's own row appended, and optionally
// w_j += sum over the unit's query heads of p_j for every cached token (its accumulated attention weight).
//
// Bound by HBM: a token of a unit costs 512 bytes (its K and V rows) and 4 g d flops.  All tokens of the layer are cut into
// tiles of 16 (never across units); the warps of a grid that fills the GPU once take equal, contiguous runs of
// tiles, whichever units they fall into, so a ragged batch and one long sequence both keep every SM busy and no
// plan on the host is needed (the lengths stay on the device and a captured call follows them).  A warp streams
// its tiles through a ring of its own in shared memory (16-byte cp.async, zero fill behind the last token) and never waits
// for another warp.  S^T = K Q^T and O^T = V^T P^T run on m16n8k16 bf16 matrix instructions with the tokens,
// respectively the channels, as the 16 rows: the 8 columns are the query heads, so nothing of the tile is padding for g = 8
// and half is for g = 4.  The fifth-generation tensor path has 128 rows per instruction and wants the whole CTA
// in step; at 4 g flops per 4 bytes it would wait for memory just the same.
// The online softmax keeps maximum and sum in fp32 (base 2).  For the product with V, whose matrix instruction takes bf16, p enters as two
// bf16 terms: its upper half and what that leaves out, together within 2^-16 of p (one term, 2^-8, showed where the values
// cancel: 13 times the error bound of the other roundings).  The second product is eight instructions per tile on a pipe that waits for memory.
//
// A second kernel joins the pieces of units that more than one warp worked on and adds the weights: the scores
// (fp32, 4 g bytes per token) wait in the workspace until the unit's sum is known.
//
// Measured (both kernels, one layer, device time of calls in a row): 8 heads x 131072 tokens, g = 5: 89.3 us = 6.0 TB/s, 0.92 of the copy
// rate; 8 heads x 16 ragged sequences (152 K tokens), g = 4, with weights: 118 us = 5.4 TB/s; 8 heads x 2458 tokens, g = 4, with
// weights: 10.9 us, the chains of two kernels (lengths, page ids, rows, one or two tiles, results; results, scores, weights).
// More than 16 query heads per KV head are served 16 at a time, and every 16 read the unit's rows again: 8 heads x 131072 tokens
// 98 us for g = 16, 172 for 32, 326 for 64.
#include "paged.cuh"

namespace compactor {
namespace {

constexpr int kTile = kDecodeTile;
constexpr int kWarps = kDecodeWarps;
constexpr int kThreads = kWarps * 32;
constexpr int kStages = 2;
constexpr int kRowBytes = kD * 2;
constexpr int kStageBytes = 2 * kTile * kRowBytes;     // K tile, V tile
constexpr size_t kSmemBytes = (size_t)kWarps * kStages * kStageBytes;
constexpr int kUnitCost = kDecodeUnitCost;
constexpr int kMassUnitCost = kDecodeMassUnitCost;
constexpr int kUnitsPerBlock = 1024;                   // most units that every joining block scans (a block of the weights scans them all, however many)
constexpr int kUnitsInSmem = 2048;                     // units whose token counts every CTA keeps at hand
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
// Two weights (0, or 2^-126 .. 1) as two pairs of bf16 terms, hi + lo.  hi is cut off, so lo is not negative, below 2^-7 of its weight's power of
// two, and rounded by at most 2^-16 of that.  lo is never 0 where the weight is not, so that a weight of an infinite value gives infinity and not
// 0 * inf in the second product; the least that it is raised to, 2^-126, is where weights end as well.
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t& hi, uint32_t& lo) {
    const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
    const float xl = fmaxf(x - __uint_as_float(xb & 0xffff0000u), fminf(x, 0x1p-126f));
    const float yl = fmaxf(y - __uint_as_float(yb & 0xffff0000u), fminf(y, 0x1p-126f));
    hi = __byte_perm(xb, yb, 0x7632);
    lo = pack_bf16(xl, yl);
}

// Tokens that a unit attends to, the new one included; 0 for a row without a sequence (negative length) and for a unit
// that would not fit (reported by the caller).
__device__ __forceinline__ int live_tokens(const DecodeArgs& a, int unit) {
    const int n = __ldcg(a.lengths + unit);
    if (n < 0) return 0;
    const long long t = (long long)n + (a.k_new != nullptr);
    return t > a.capacity ? 0 : (int)t;
}
__device__ __forceinline__ int tiles_of(int tokens) { return (tokens + kTile - 1) / kTile; }
// What a (unit, group) counts for when the work is shared out: its tiles and kUnitCost more, since a warp that enters
// a unit waits for its queries, page ids and row of results (with 0 the warps that got many short units of a padded batch ended
// last: the first kernel took 36 us instead of 22).
__device__ __forceinline__ int cost_of(int tokens) { return tokens == 0 ? 0 : tiles_of(tokens) + kUnitCost; }

// `total` cost shared by `workers`: the first total % workers get one more than the others.
struct Share {
    int q, r;
    __device__ __forceinline__ Share(int total, int workers) : q(total / workers), r(total - total / workers * workers) {}
    __device__ __forceinline__ int begin(int w) const { return w * q + min(w, r); }
    __device__ __forceinline__ int size(int w) const { return q + (w < r ? 1 : 0); }
    __device__ __forceinline__ int owner(int at) const {
        const int longer = r * (q + 1);
        return at < longer ? at / (q + 1) : r + (at - longer) / q;
    }
};
// Warps that share the work.  Where each gets many tiles one warp of a CTA stays out: with seven warps of two stages 112 KB are on
// their way to an SM, enough for its share of HBM; more of them disturb each other (131072 tokens: 88.9 us with seven warps, 89.1
// with eight, 96.4 with eight of three stages, 90.1 with six).  With few tiles all eight are wanted (padded batch: 31.8 against 33.1 us).
__device__ __forceinline__ int active_workers(const DecodeArgs& a, int total) {
    return total / 16 >= a.workers ? a.workers / kWarps * (kWarps - 1) : min(a.workers, total);
}

// A place in the order of all tiles: unit by unit, within a unit group by group.
struct Cursor {
    int unit, grp, tile, tiles, tokens;
    // Next (unit, group) that has tiles; false if there is none.
    __device__ __forceinline__ bool next_unit(const DecodeArgs& a, const int* live) {
        tile = 0;
        if (grp + 1 < a.groups) { ++grp; return true; }
        grp = 0;
        do {
            if (++unit >= a.units) return false;
            tokens = unit < kUnitsInSmem ? live[unit] : live_tokens(a, unit);
        } while (tokens == 0);
        tiles = tiles_of(tokens);
        return true;
    }
};

// Page ids of a unit, entry `e0 + lane` of its row of the table (-1 behind its last token's).
__device__ __forceinline__ int page_ids(const DecodeArgs& a, const Cursor& c, int e0, int lane) {
    const int e = e0 + lane;
    return e <= (c.tokens - 1) >> a.c.page_shift ? __ldcg(a.c.table + (long long)c.unit * a.c.max_pages + e) : -1;
}

// Query fragments (B operand) of a unit's group: head t * 8 + gid, channels 16 s + 2 tig, + 1 and + 8, + 9.
template <int NG>
__device__ __forceinline__ void load_queries(const DecodeArgs& a, const Cursor& c, uint32_t (&qf)[NG][8][2], int lane) {
    const int gid = lane >> 2, tig = lane & 3;
    const int h = c.unit / a.c.batch, b = c.unit - h * a.c.batch;
    const int head0 = h * a.g + c.grp * kDecodeHeads, heads = min(kDecodeHeads, a.g - c.grp * kDecodeHeads);
#pragma unroll
    for (int t = 0; t < NG; ++t) {
        const bool on = t * 8 + gid < heads;
        const uint32_t* q = reinterpret_cast<const uint32_t*>(a.q + b * a.q_seq + (long long)(head0 + (on ? t * 8 + gid : 0)) * a.q_head);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const uint32_t x0 = q[s * 8 + tig], x1 = q[s * 8 + tig + 4];
            qf[t][s][0] = on ? x0 : 0u;
            qf[t][s][1] = on ? x1 : 0u;
        }
    }
}

template <int NG>
__global__ void __launch_bounds__(kThreads, 1)
decode_kernel(const __grid_constant__ DecodeArgs a) {
    extern __shared__ __align__(1024) unsigned char ring[];
    __shared__ int cum[kThreads + 1];
    __shared__ int warp_sum[kWarps];
    __shared__ int bad[kWarps][kStages];
    __shared__ int new_page[kWarps][kStages];
    __shared__ int live[kUnitsInSmem];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    pdl_wait();

    // cost before each thread's run of units
    const int per = (a.units + kThreads - 1) / kThreads;
    const int u0 = tid * per, u1 = min(a.units, u0 + per);
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

    // ---- producer: one tile into a stage.  Lane l copies 16-byte piece l & 15 of rows (l >> 4) + 2 i.  What the next tiles
    // need is asked for early: 64 page ids of the unit (lane l holds entries e0 + l and e0 + 32 + l), the first 32 of the unit
    // after it, and the queries of a unit when its first tile is issued.
    Cursor pc = start, nc = start;
    const int piece = lane & 15, row_hi = lane >> 4;
    int e0 = (pc.tile * kTile) >> a.c.page_shift;
    int ids = page_ids(a, pc, e0, lane), ids_after = page_ids(a, pc, e0 + 32, lane), ids_next_unit = -1;
    uint32_t qn[NG][8][2];
    int q_unit = pc.unit, q_grp = pc.grp;                    // whose queries qn holds
    bool q_waiting = true;
    load_queries<NG>(a, pc, qn, lane);
    if (nc.next_unit(a, live)) ids_next_unit = page_ids(a, nc, 0, lane);
    // Eight rows to `dst` (and the same of V a tile further) from `src`, this lane's piece of the run's first or second row on.  Row r's pieces stand in
    // the stage with their number xor r & 7, so that the eight rows of a matrix fragment meet different banks.
    const long long two_rows = 2 * a.c.stride_token * (long long)sizeof(__nv_bfloat16);
    const long long v_from_k = reinterpret_cast<const char*>(a.c.v) - reinterpret_cast<const char*>(a.c.k);
    uint32_t place[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) place[i] = (2 * i + row_hi) * kRowBytes + ((piece ^ (2 * i + row_hi)) << 4);
    auto copy_rows = [&](uint32_t dst, const char* src) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cp_async16(dst + place[i], src);
            cp_async16(dst + place[i] + kTile * kRowBytes, src + v_from_k);
            src += two_rows;
        }
    };
    int in_stage = 0;
    auto issue = [&]() {
        if (left_p > 0) {
            const int stage = in_stage;
            const int unit = pc.unit, n = pc.tokens, base = pc.tile * kTile;
            const int cached = n - (a.k_new != nullptr);     // tokens whose rows are in pages
            const int e = base >> a.c.page_shift;
            if (e + 1 >= e0 + 32) {                          // (pages of 8 tokens: a tile has two)
                e0 += 32;
                if (e < e0) {                                // a tile on the seam keeps one entry of the old run
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
            int p0 = __shfl_sync(0xffffffffu, ids, e - e0), p1 = __shfl_sync(0xffffffffu, ids, ((base + 8) >> a.c.page_shift) - e0);
            if ((unsigned)p0 >= (unsigned)a.c.n_pages) p0 = -1;
            if ((unsigned)p1 >= (unsigned)a.c.n_pages || base + 8 >= n) p1 = -1;
            const uint32_t ks = ring_s + stage * kStageBytes;
            const int fresh_row = cached < n ? cached - base : -1;           // the new token's row of this tile, if it has it
            if (base + kTile <= cached && p0 >= 0 && p1 >= 0) {              // all rows come from pages: two runs of eight
                const char* src = reinterpret_cast<const char*>(a.c.k + row_in_pool(a.c, p0, base + row_hi)) + piece * 16;
                copy_rows(ks, src);
                src = reinterpret_cast<const char*>(a.c.k + row_in_pool(a.c, p1, base + 8 + row_hi)) + piece * 16;
                copy_rows(ks + 8 * kRowBytes, src);
            } else {
                const int h = unit / a.c.batch, b = unit - h * a.c.batch;
#pragma unroll 1
                for (int i = 0; i < kTile / 2; ++i) {
                    const int row = 2 * i + row_hi, tok = base + row;
                    const int page = i < kTile / 4 ? p0 : p1;
                    const bool is_new = row == fresh_row, on = is_new || (tok < cached && page >= 0);
                    const long long off = on && !is_new ? row_in_pool(a.c, page, tok) + piece * 8 : 0;
                    const __nv_bfloat16* kr = is_new ? a.k_new + b * a.kn_seq + h * a.kn_head + piece * 8 : a.c.k + off;
                    const __nv_bfloat16* vr = is_new ? a.v_new + b * a.vn_seq + h * a.vn_head + piece * 8 : a.c.v + off;
                    const uint32_t dst = ks + row * kRowBytes + ((piece ^ (row & 7)) << 4);
                    cp_async16(dst, kr, on ? 16 : 0);
                    cp_async16(dst + kTile * kRowBytes, vr, on ? 16 : 0);
                }
            }
            if (lane == 0) {
                const int bits = (p0 < 0 && base < cached ? 1 : 0) | (p1 < 0 && base + 8 < cached ? 2 : 0);
                const int np = fresh_row < 8 ? p0 : p1;
                bad[warp][stage] = bits;
                new_page[warp][stage] = np;
                if (a.status != nullptr && (bits != 0 || (fresh_row >= 0 && fresh_row < kTile && np < 0)))
                    atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
            }
            in_stage = stage + 1 == kStages ? 0 : stage + 1;
            --left_p;
            if (++pc.tile == pc.tiles && (left_p -= kUnitCost) > 0) {
                pc = nc;
                e0 = 0;
                ids = ids_next_unit;
                ids_after = page_ids(a, pc, 32, lane);
                if (nc.next_unit(a, live)) ids_next_unit = page_ids(a, nc, 0, lane);
                if (!q_waiting) {
                    load_queries<NG>(a, pc, qn, lane);
                    q_unit = pc.unit; q_grp = pc.grp; q_waiting = true;
                }
            }
        }
        cp_commit();
    };
#pragma unroll 1
    for (int s = 0; s < kStages; ++s) issue();

    // ---- consumer
    // fragment s of a row: pieces 2 s and 2 s + 1, i.e. (piece ^ r & 7) << 4 = place of piece 0 or 1, xor s << 5 (a stage starts at a multiple of 256)
    const uint32_t k_frag = ((lane & 7) + ((lane >> 3) & 1) * 8) * kRowBytes + (((lane >> 4) ^ (lane & 7)) << 4);
    const uint32_t v_frag = ((lane & 7) + (lane >> 4) * 8) * kRowBytes + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
    Cursor cc = start;
    const float scale2 = a.scale * kLog2e;
    const float cap_in = a.softcap > 0.f ? a.scale / a.softcap : 0.f, cap_out = a.softcap * kLog2e;
    uint32_t qf[NG][8][2];
    float o[NG][8][4];
    float mx[NG][2], sum[NG][2];
    bool fresh = true;
    int first_tile = 0, head0 = 0, heads = 0, stage = 0;

    while (true) {
        if (fresh) {                                         // a new unit or group: its queries
            fresh = false;
            first_tile = cc.tile;
            head0 = cc.unit / a.c.batch * a.g + cc.grp * kDecodeHeads;
            heads = min(kDecodeHeads, a.g - cc.grp * kDecodeHeads);
            if (q_waiting && q_unit == cc.unit && q_grp == cc.grp) {
                q_waiting = false;
#pragma unroll
                for (int t = 0; t < NG; ++t)
#pragma unroll
                    for (int s = 0; s < 8; ++s) { qf[t][s][0] = qn[t][s][0]; qf[t][s][1] = qn[t][s][1]; }
            } else {
                load_queries<NG>(a, cc, qf, lane);
            }
#pragma unroll
            for (int t = 0; t < NG; ++t) {
#pragma unroll
                for (int s = 0; s < 8; ++s) o[t][s][0] = o[t][s][1] = o[t][s][2] = o[t][s][3] = 0.f;
                mx[t][0] = mx[t][1] = -INFINITY;
                sum[t][0] = sum[t][1] = 0.f;
            }
        }
        // the second kernel's blocks are let in when the tiles run out: let in at the start they gain nothing (47.7 us either way for 8
        // sequences x 4 heads x 7 queries) and hold registers of every SM all the while
        if (left_c <= kStages) pdl_trigger();
        cp_wait<kStages - 1>();
        __syncwarp();
        const uint32_t ks = ring_s + stage * kStageBytes, vs = ks + kTile * kRowBytes;
        const int base = cc.tile * kTile;

        // S^T: 16 tokens x 8 NG heads
        float s[NG][4];
#pragma unroll
        for (int t = 0; t < NG; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
        {
#pragma unroll
            for (int st = 0; st < 8; ++st) {
                uint32_t kf[4];
                ldsm4(kf, (ks + k_frag) ^ (st << 5));
#pragma unroll
                for (int t = 0; t < NG; ++t) mma(s[t], kf, qf[t][st][0], qf[t][st][1]);
            }
        }
        // scores in base 2; what does not count gets -inf
        const int bits = bad[warp][stage];
        const int cached = cc.tokens - (a.k_new != nullptr);
        const int ta = base + gid, tb = ta + 8;
        const bool la = ta < cc.tokens && !((bits & 1) && ta < cached), lb = tb < cc.tokens && !((bits & 2) && tb < cached);
        uint32_t pf[NG][2], pl[NG][2];                       // weights: first and second term
        bool grew = false;
        float scale_by[NG][2];
#pragma unroll
        for (int t = 0; t < NG; ++t) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float y = a.softcap > 0.f ? cap_out * tanhf(s[t][c] * cap_in) : s[t][c] * scale2;
                s[t][c] = (c < 2 ? la : lb) ? y : -INFINITY;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float m = fmaxf(s[t][c], s[t][c + 2]);
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                m = fmaxf(m, mx[t][c]);
                grew |= m > mx[t][c];
                const float ref = m == -INFINITY ? 0.f : m;
                scale_by[t][c] = ex2f(mx[t][c] - ref);       // 0 for the first tile, 1 where the maximum stays
                mx[t][c] = m;
                const float pa = ex2f(s[t][c] - ref), pb = ex2f(s[t][c + 2] - ref);
                sum[t][c] = sum[t][c] * scale_by[t][c] + (pa + pb);
                if (c == 0) { pf[t][0] = __float_as_uint(pa); pf[t][1] = __float_as_uint(pb); }
                else {
                    split_bf16(__uint_as_float(pf[t][0]), pa, pf[t][0], pl[t][0]);
                    split_bf16(__uint_as_float(pf[t][1]), pb, pf[t][1], pl[t][1]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) { pf[t][i] = transpose8x8(pf[t][i]); pl[t][i] = transpose8x8(pl[t][i]); }
        }
        if (a.accumulate) {                                  // kept until the sum over the whole unit is known
            float* col = a.scores + ((long long)cc.unit * a.g + cc.grp * kDecodeHeads + 2 * tig) * a.unit_rows + base + gid;
#pragma unroll
            for (int t = 0; t < NG; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (t * 8 + 2 * tig + c < heads) {       // 32 bytes of a head's scores per group of eight lanes
                        float* at = col + (long long)(t * 8 + c) * a.unit_rows;
                        at[0] = s[t][c];
                        at[8] = s[t][c + 2];
                    }
        }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int t = 0; t < NG; ++t)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    o[t][j][0] *= scale_by[t][0]; o[t][j][1] *= scale_by[t][1];
                    o[t][j][2] *= scale_by[t][0]; o[t][j][3] *= scale_by[t][1];
                }
        }
        // O^T += V^T P^T: 128 channels x 8 NG heads
        {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t vf[4];
                ldsm4t(vf, (vs + v_frag) ^ (j << 5));
#pragma unroll
                for (int t = 0; t < NG; ++t) mma(o[t][j], vf, pf[t][0], pf[t][1]);
#pragma unroll
                for (int t = 0; t < NG; ++t) mma(o[t][j], vf, pl[t][0], pl[t][1]);
            }
        }
        // the new token's row goes from the ring to its page
        const int fresh_row = cached < cc.tokens && cc.grp == 0 ? cached - base : -1;
        if (fresh_row >= 0 && fresh_row < kTile) {
            const int page = new_page[warp][stage];
            if (page >= 0) {
                const uint4 x = *reinterpret_cast<const uint4*>(my_ring + stage * kStageBytes + row_hi * (kTile * kRowBytes) +
                                                                fresh_row * kRowBytes + ((piece ^ (fresh_row & 7)) << 4));
                *reinterpret_cast<uint4*>((row_hi == 0 ? a.c.k : a.c.v) + row_in_pool(a.c, page, cached) + piece * 8) = x;
                const long long at = slot_in_pool(a.c, page, cached);
                if (lane == 0 && a.c.positions != nullptr)
                    a.c.positions[at] = a.new_positions != nullptr ? a.new_positions[cc.unit % a.c.batch] : cached;
                if (lane == 0 && a.c.mass != nullptr && !a.accumulate) a.c.mass[at] = 0.f;
            }
        }
        __syncwarp();
        issue();

        stage = stage + 1 == kStages ? 0 : stage + 1;
        --left_c;
        const bool unit_ends = ++cc.tile == cc.tiles;
        if (unit_ends) left_c -= kUnitCost;
        if (unit_ends || left_c <= 0) {                   // hand over what this warp has of the unit
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
                        a.ml[slot * 32 + head] = mx[t][c];
                        a.ml[slot * 32 + 16 + head] = l;
                    }
                    if (whole) {
                        const float inv = l == 0.f ? 0.f : 1.f / l;
                        __nv_bfloat16* dst = a.out + b * a.out_seq + (long long)(head0 + head) * a.out_head + gid;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            dst[16 * j] = __float2bfloat16_rn(o[t][j][c] * inv);
                            dst[16 * j + 8] = __float2bfloat16_rn(o[t][j][c + 2] * inv);
                        }
                        if (gid == 0 && a.lse != nullptr)
                            a.lse[(long long)b * (a.c.heads * a.g) + head0 + head] = l == 0.f ? -INFINITY : kLn2 * (mx[t][c] + log2f(l));
                    } else {
                        float* dst = a.o + (slot * gg + head) * kD + gid;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            dst[16 * j] = o[t][j][c];
                            dst[16 * j + 8] = o[t][j][c + 2];
                        }
                    }
                }
            if (left_c <= 0) return;
            fresh = true;
            cc.next_unit(a, live);
        }
    }
}

// Running (max, sum) in base 2.
__device__ __forceinline__ void merge(float& m, float& l, float mo, float lo) {
    const float mm = fmaxf(m, mo);
    const float ref = mm == -INFINITY ? 0.f : mm;
    l = l * ex2f(m - ref) + lo * ex2f(mo - ref);
    m = mm;
}

// The pieces of a unit's group: partial slots [first, first + n).  `at`, `cost`: the unit's place and its cost per group.
struct Pieces { long long first; int n; };
__device__ __forceinline__ Pieces pieces_of(const DecodeArgs& a, int unit, int grp, int at, int cost, int all) {
    const int total = all * a.groups;
    const Share share(total, active_workers(a, total));
    const int v = at * a.groups + grp * cost;
    const int w0 = share.owner(v + kUnitCost), w1 = share.owner(v + cost - 1);
    return {(long long)w0 + (long long)unit * a.groups + grp, w1 - w0 + 1};
}

// The last blocks have kItems (unit, query head) pairs each, whose pieces they join: o = sum_i e_i o_i / sum_i e_i l_i with
// e_i = 2^(m_i - m).  The blocks before them add the weights; they share all tokens out evenly, as the first kernel does,
// with a cost of kMassUnitCost tiles per unit (about what its sum takes to find).  Both are chains of a few dependent reads from L2
// (about 0.7 us each), so every step asks for all it needs at once, and several small blocks share an SM.
template <int kWarps, int kItems>
__global__ void __launch_bounds__(kWarps * 32, kWarps == 16 ? 1 : 4)
join_kernel(const __grid_constant__ DecodeArgs a, int mass_blocks) {
    constexpr int kThreads = kWarps * 32;
    constexpr int kJoinBatch = kWarps == 16 ? 8 : 4;         // pieces per warp in flight
    // a large block takes half of the channels of its (unit, head): twice as many pieces in flight per warp
    constexpr int kSplit = kWarps == 16 ? 2 : 1, kLanes = 32 / kSplit, kChannels = kD / kSplit;
    constexpr int kItemWarps = kWarps / kItems, kStreams = kItemWarps * kSplit;
    static_assert(kItems == 1 || kSplit == 1, "a block has several pairs or half of one");
    __shared__ float part[kItems * kStreams][kChannels];
    __shared__ float part_m[kItems * kStreams], part_l[kItems * kStreams];
    __shared__ bool to_write[kItems];
    __shared__ float red_m[kWarps][16], red_l[kWarps][16];
    __shared__ float lse2[64];
    __shared__ long long sums[kWarps];
    __shared__ int found[3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // Until pdl_wait() nothing of the first kernel's is read: what depends on lengths, pages and old weights alone (they were there
    // before it began, and are read from L2) is worked out while its last warps finish.  No block ends before pdl_wait(): the next launch counts on both kernels being done.
    if (kWarps == 16) pdl_trigger();                         // (else the next call's blocks would take the registers of the later blocks of this one)
    if ((int)blockIdx.x >= mass_blocks) {
        const int nth = warp / kItemWarps, warp_of_item = warp - nth * kItemWarps;
        const int item = (blockIdx.x - mass_blocks) / kSplit * kItems + nth, unit = min(item / a.g, a.units - 1);
        const int channel0 = ((blockIdx.x - mass_blocks) % kSplit) * kChannels;
        const int head = item - unit * a.g, grp = head / kDecodeHeads, hh = head - grp * kDecodeHeads, gg = min(a.g, kDecodeHeads);
        int at, cost, all;                                   // the unit's place and cost, the cost of all units
        if (a.units <= kUnitsPerBlock) {
            long long x = 0;                                 // cost before the unit, and in the upper half of all
            for (int u = warp_of_item * 32 + lane; u < a.units; u += kItemWarps * 32) {
                const int c = cost_of(live_tokens(a, u));
                x += ((long long)c << 32) + (u < unit ? c : 0);
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            if (lane == 0) sums[warp] = x;
            __syncthreads();
            x = 0;
#pragma unroll
            for (int w = 0; w < kItemWarps; ++w) x += sums[nth * kItemWarps + w];
            at = (int)x; all = (int)(x >> 32); cost = cost_of(live_tokens(a, unit));
            pdl_wait();
        } else {                                             // the first kernel's prefix, so that the many blocks need not scan the many units
            pdl_wait();
            at = a.prefix[unit]; cost = a.prefix[unit + 1] - at; all = a.prefix[a.units];
        }
        // an empty unit: nothing to add up, which gives a zero row and lse = -inf; a unit of one piece was written by the warp that had it
        Pieces ps = {0, 0};
        if (cost > 0) ps = pieces_of(a, unit, grp, at, cost, all);
        const bool write = item < a.units * a.g && ps.n != 1;
        if (kItems == 1 && !write) return;
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        const int stream = warp_of_item * kSplit + lane / kLanes, channel = lane % kLanes * 4;
        for (int i0 = stream; write && i0 < ps.n; i0 += kStreams * kJoinBatch) {
            float pm[kJoinBatch], pl[kJoinBatch];
            float4 x[kJoinBatch];
#pragma unroll
            for (int k = 0; k < kJoinBatch; ++k) {
                const long long slot = ps.first + min(i0 + k * kStreams, ps.n - 1);
                pm[k] = a.ml[slot * 32 + hh];
                pl[k] = a.ml[slot * 32 + 16 + hh];
                x[k] = *reinterpret_cast<const float4*>(a.o + (slot * gg + hh) * kD + channel0 + channel);
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < kJoinBatch; ++k) {
                if (i0 + k * kStreams >= ps.n) pm[k] = -INFINITY;
                top = fmaxf(top, pm[k]);
            }
            const float ref = top == -INFINITY ? 0.f : top;
            const float old = ex2f(m - ref);
            l *= old; acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
            m = top;
#pragma unroll
            for (int k = 0; k < kJoinBatch; ++k) {
                if (i0 + k * kStreams >= ps.n) continue;
                const float e = ex2f(pm[k] - ref);
                l += e * pl[k];
                acc.x += e * x[k].x; acc.y += e * x[k].y; acc.z += e * x[k].z; acc.w += e * x[k].w;
            }
        }
        *reinterpret_cast<float4*>(&part[nth * kStreams + stream][channel]) = acc;
        if (channel == 0) { part_m[nth * kStreams + stream] = m; part_l[nth * kStreams + stream] = l; }
        if (lane == 0) to_write[nth] = write;
        __syncthreads();
        for (int i = tid; i < kItems * kChannels; i += kThreads) {
            const int which = i / kChannels, ch = i % kChannels, first = which * kStreams;
            if (!to_write[which]) continue;
            const int pair = (blockIdx.x - mass_blocks) / kSplit * kItems + which, u = pair / a.g;
            const int h = u / a.c.batch, b = u - h * a.c.batch, q_head = h * a.g + pair - u * a.g;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kStreams; ++w) top = fmaxf(top, part_m[first + w]);
            const float ref = top == -INFINITY ? 0.f : top;
            float x = 0.f, z = 0.f;
#pragma unroll
            for (int w = 0; w < kStreams; ++w) {
                const float e = ex2f(part_m[first + w] - ref);
                x += e * part[first + w][ch];
                z += e * part_l[first + w];
            }
            a.out[b * a.out_seq + (long long)q_head * a.out_head + channel0 + ch] = __float2bfloat16_rn(z == 0.f ? 0.f : x / z);
            if (channel0 + ch == 0 && a.lse != nullptr)
                a.lse[(long long)b * (a.c.heads * a.g) + q_head] = z == 0.f ? -INFINITY : kLn2 * (top + log2f(z));
        }
        return;
    }

    // weights: w_j += sum over the unit's query heads of 2^(y_j - lse)
    int unit, at, place_of_unit, all;                        // the unit that holds this block's first place, its place for the tiles and for the weights
    int place, place_end;
    {
        const int per = (a.units + kThreads - 1) / kThreads, u0 = tid * per, u1 = min(a.units, u0 + per);
        long long mine = 0;                                  // cost, and in the upper half how many units have tokens
        for (int u = u0; u < u1; ++u) {
            const int n = live_tokens(a, u);
            mine += cost_of(n) + ((long long)(n > 0) << 32);
        }
        long long incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += o;
        }
        if (lane == 31) sums[warp] = incl;
        __syncthreads();
        long long before = incl - mine, total = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sums[w];
            total += sums[w];
        }
        constexpr int kMore = kMassUnitCost - kUnitCost;
        all = (int)total;
        const Share share(all + (int)(total >> 32) * kMore, mass_blocks);
        place = share.begin(blockIdx.x);
        place_end = place + share.size(blockIdx.x);
        int my_at = (int)before, my_place = my_at + (int)(before >> 32) * kMore;
        for (int u = u0; u < u1; ++u) {
            const int c = cost_of(live_tokens(a, u));
            if (c == 0) continue;
            if (my_place <= place && place < my_place + c + kMore) { found[0] = u; found[1] = my_at; found[2] = my_place; }
            my_at += c; my_place += c + kMore;
        }
        __syncthreads();
        if (place >= place_end) { pdl_wait(); return; }
        unit = found[0]; at = found[1]; place_of_unit = found[2];
    }
    int hp = 1;                                              // lanes side by side for the heads of a group
    while (hp < min(a.g, kDecodeHeads)) hp *= 2;
    const int hh = lane & (hp - 1), st = tid / hp, streams = kThreads / hp;
    for (; place < place_end; ++unit) {
        const int n = live_tokens(a, unit), cost = cost_of(n);
        if (n == 0) continue;
        const int here = at, first_place = place_of_unit + kMassUnitCost;
        at += cost;
        place_of_unit += tiles_of(n) + kMassUnitCost;
        const int first_tile = max(0, place - first_place), last_tile = min(place_end, place_of_unit) - first_place;
        place = place_of_unit;
        if (last_tile <= first_tile) continue;               // only the unit's head
        const int tok0 = first_tile * kTile, tok1 = min(n, last_tile * kTile);
        const int cached = n - (a.k_new != nullptr);
        // four tokens a thread: they share a page and a 16-byte piece of its weights
        int page;
        float4 old;
        auto ask_page = [&](int first) { page = page_of<true>(a.c, unit, min(first, (tok1 - 1) & ~3)); };
        auto ask_weights = [&](int first) {
            old = __ldcg(reinterpret_cast<const float4*>(a.c.mass + slot_in_pool(a.c, max(page, 0), min(first, (tok1 - 1) & ~3))));
        };
        ask_page(tok0 + 4 * tid);
        ask_weights(tok0 + 4 * tid);
        pdl_wait();
        for (int grp = 0; grp < a.groups; ++grp) {
            const Pieces ps = pieces_of(a, unit, grp, here, cost, all);
            const int heads = min(kDecodeHeads, a.g - grp * kDecodeHeads);
            float m = -INFINITY, l = 0.f;
            if (hh < heads) {
#pragma unroll 4
                for (int i = st; i < ps.n; i += streams) {
                    const float* ml = a.ml + (ps.first + i) * 32 + hh;
                    merge(m, l, ml[0], ml[16]);
                }
            }
            // the block's maximum per head, then the sums against it: a tree of single shuffles each, then one round over the warps
            float top = m;
            for (int d = hp; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            l *= ex2f(m - (top == -INFINITY ? 0.f : top));
            for (int d = hp; d < 32; d *= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
            if (lane < hp) { red_m[warp][lane] = top; red_l[warp][lane] = l; }
            __syncthreads();
            if (tid < heads) {
                top = red_m[0][tid];
#pragma unroll
                for (int i = 1; i < kWarps; ++i) top = fmaxf(top, red_m[i][tid]);
                const float ref = top == -INFINITY ? 0.f : top;
                l = 0.f;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) l += red_l[i][tid] * ex2f(red_m[i][tid] - ref);
                lse2[grp * kDecodeHeads + tid] = l == 0.f ? INFINITY : top + log2f(l);
            }
            __syncthreads();
        }
        for (int first = tok0 + 4 * tid; first < tok1; first += 4 * kThreads) {
            float w[4] = {};
            const float* col = a.scores + (long long)unit * a.g * a.unit_rows + first;
#pragma unroll 4
            for (int i = 0; i < a.g; ++i, col += a.unit_rows) {
                const float4 y = *reinterpret_cast<const float4*>(col);
                const float z = lse2[i];
                w[0] += ex2f(y.x - z); w[1] += ex2f(y.y - z); w[2] += ex2f(y.z - z); w[3] += ex2f(y.w - z);
            }
            if (page >= 0) {
                float* at_mass = a.c.mass + slot_in_pool(a.c, page, first);
                if (first + 4 <= min(tok1, cached)) {
                    *reinterpret_cast<float4*>(at_mass) = make_float4(old.x + w[0], old.y + w[1], old.z + w[2], old.w + w[3]);
                } else {
                    const float o[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (first + k < tok1) at_mass[k] = first + k < cached ? o[k] + w[k] : w[k];
                }
            }
            if (first + 4 * kThreads < tok1) {
                ask_page(first + 4 * kThreads);
                ask_weights(first + 4 * kThreads);
            }
        }
        __syncthreads();                                     // lse2 and the reductions are the next unit's
    }
    pdl_wait();                                              // (a block that met only heads of units has not waited yet)
}

}  // namespace

cudaError_t launch_paged_attention(const DecodeArgs& a, int sm_count, cudaStream_t stream) {
    const int grid = a.workers / kWarps;
    static std::atomic<unsigned long long> done[2];
    auto kernel = a.g <= 8 ? decode_kernel<1> : decode_kernel<2>;
    cudaError_t e = allow_smem(kernel, (int)kSmemBytes, done[a.g <= 8 ? 0 : 1]);
    if (e != cudaSuccess) return e;
    if ((e = launch_chained(kPdlOther, kernel, dim3(grid), dim3(kThreads), kSmemBytes, stream, a)) != cudaSuccess) return e;
    // the second kernel.  Few (unit, head) pairs: 16 warps a block and two blocks per pair, where all of them fit the GPU at once, one to
    // an SM.  More: 8 warps a block, four blocks to an SM; with few pieces a pair, four pairs a block.
    const int pairs = a.units * a.g;
    const long long most = a.accumulate ? (long long)a.units * ((a.capacity + kTile - 1) / kTile + kMassUnitCost) : 0;   // cost of the weights
    const long long wanted = (most + kTile - 1) / kTile;     // 256 tokens a block at the least
    const bool large = 2 * pairs <= sm_count, few_pieces = a.workers < 6 * a.units * a.groups;
    const int join_blocks = large ? 2 * pairs : few_pieces ? (pairs + 3) / 4 : pairs;
    // (not more than fit beside the others, so that those need not wait for a place)
    const int room = large ? max(sm_count / 2, sm_count - join_blocks) : join_blocks <= 2 * sm_count ? 4 * sm_count - join_blocks : 4 * sm_count;
    const int mass_blocks = (int)min(wanted, (long long)room);
    const dim3 blocks(mass_blocks + join_blocks);
    e = large        ? launch_chained(kPdlOther, join_kernel<16, 1>, blocks, dim3(512), 0, stream, a, mass_blocks)
        : few_pieces ? launch_chained(kPdlOther, join_kernel<8, 4>, blocks, dim3(256), 0, stream, a, mass_blocks)
                     : launch_chained(kPdlOther, join_kernel<8, 1>, blocks, dim3(256), 0, stream, a, mass_blocks);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace compactor
