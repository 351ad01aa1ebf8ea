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
// The online softmax keeps maximum and sum in fp32 (base 2); p is rounded to bf16 for the product with V (at most 2^-9
// relative per weight, the sum uses the unrounded values).
//
// A second kernel joins the pieces of units that more than one warp worked on and adds the weights: the scores
// (fp32, 4 g bytes per token) wait in the workspace until the unit's sum is known.
#include "paged.cuh"

namespace compactor {
namespace {

constexpr int kTile = kDecodeTile;
constexpr int kWarps = kDecodeWarps;
constexpr int kThreads = kWarps * 32;
constexpr int kStages = 3;
constexpr int kRowBytes = kD * 2;
constexpr int kStageBytes = 2 * kTile * kRowBytes;     // K tile, V tile
constexpr size_t kSmemBytes = (size_t)kWarps * kStages * kStageBytes;
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

// Tokens that a unit attends to, the new one included; 0 for a row without a sequence (negative length) and for a unit
// that would not fit (reported by the caller).
__device__ __forceinline__ int live_tokens(const DecodeArgs& a, int unit) {
    const int n = __ldg(a.lengths + unit);
    if (n < 0) return 0;
    const long long t = (long long)n + (a.k_new != nullptr);
    return t > a.capacity ? 0 : (int)t;
}
__device__ __forceinline__ int tiles_of(int tokens) { return (tokens + kTile - 1) / kTile; }

// Worker that owns tile t of `total` tiles shared by `workers` workers, worker w having [w total / workers, (w+1) total / workers).
__device__ __forceinline__ int owner(long long t, long long total, long long workers) {
    return (int)(((t + 1) * workers - 1) / total);
}

// A place in the order of all tiles: unit by unit, within a unit group by group.
struct Cursor {
    int unit, grp, tile, tiles, tokens;
    int before;                                              // tiles of the units before this one
    // Next (unit, group) that has tiles.  Only called while tiles remain, so it ends.
    __device__ __forceinline__ void next_unit(const DecodeArgs& a) {
        tile = 0;
        if (grp + 1 < a.groups) { ++grp; return; }
        grp = 0;
        before += tiles;
        do {
            ++unit;
            tokens = unit < a.units ? live_tokens(a, unit) : 1;
        } while (tokens == 0);
        tiles = tiles_of(tokens);
    }
};

template <int NG>
__global__ void __launch_bounds__(kThreads, 1)
decode_kernel(const __grid_constant__ DecodeArgs a) {
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ int cum[kThreads + 1];
    __shared__ int warp_sum[kWarps];
    __shared__ int bad[kWarps][kStages];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    pdl_trigger();

    // tiles before each thread's run of units
    const int per = (a.units + kThreads - 1) / kThreads;
    const int u0 = tid * per, u1 = min(a.units, u0 + per);
    int mine = 0;
    for (int u = u0; u < u1; ++u) mine += tiles_of(live_tokens(a, u));
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
    const int real_tiles = cum[kThreads];
    if (blockIdx.x == 0) {                                   // for the second kernel, and the units that are refused
        int at = cum[tid];
        for (int u = u0; u < u1; ++u) {
            a.prefix[u] = at;
            at += tiles_of(live_tokens(a, u));
            const int n = __ldg(a.lengths + u);
            if (a.status != nullptr && n >= 0 && (long long)n + (a.k_new != nullptr) > a.capacity)
                atomicOr(a.status + u, COMPACTOR_STATUS_CAPACITY);
        }
        if (tid == 0) a.prefix[a.units] = real_tiles;
    }
    const long long total = (long long)real_tiles * a.groups;
    const int workers = (int)min((long long)a.workers, total);
    const int worker = warp * gridDim.x + blockIdx.x;        // neighbouring workers on different SMs: a small call uses them all
    if (worker >= workers) return;
    const long long t0 = worker * total / workers, t1 = (worker + 1) * total / workers;
    const int count = (int)(t1 - t0);

    // the unit that holds tile t0
    Cursor start;
    {
        int lo = 0, hi = kThreads;                           // cum[lo] * groups <= t0 < cum[hi] * groups
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((long long)cum[mid] * a.groups <= t0) lo = mid; else hi = mid;
        }
        long long left = t0 - (long long)cum[lo] * a.groups;
        int u = lo * per, n = live_tokens(a, u);
        while (left >= (long long)tiles_of(n) * a.groups) {
            left -= (long long)tiles_of(n) * a.groups;
            n = live_tokens(a, ++u);
        }
        start.unit = u; start.tokens = n; start.tiles = tiles_of(n);
        start.before = (int)((t0 - left) / a.groups);
        start.grp = (int)(left / start.tiles);
        start.tile = (int)(left - (long long)start.grp * start.tiles);
    }

    unsigned char* my_ring = ring + (size_t)warp * kStages * kStageBytes;
    const uint32_t ring_s = smem_u32(my_ring);

    // ---- producer: one tile into a stage.  Lane l copies 16-byte piece l & 15 of rows (l >> 4) + 2 i.
    Cursor pc = start;
    int issued = 0;
    const int piece = lane & 15, row_hi = lane >> 4;
    auto issue = [&]() {
        if (issued < count) {
            const int stage = issued % kStages;
            const int unit = pc.unit, n = pc.tokens, base = pc.tile * kTile;
            const int cached = n - (a.k_new != nullptr);     // tokens whose rows are in pages
            const int p0 = page_of(a.c, unit, base);
            const int p1 = base + 8 < n ? page_of(a.c, unit, base + 8) : -1;
            const uint32_t ks = ring_s + stage * kStageBytes, vs = ks + kTile * kRowBytes;
            const int batch = a.c.batch, h = unit / batch, b = unit - h * batch;
#pragma unroll
            for (int i = 0; i < kTile / 2; ++i) {
                const int row = 2 * i + row_hi, tok = base + row;
                const int page = i < kTile / 4 ? p0 : p1;
                const __nv_bfloat16* ksrc = a.c.k;
                const __nv_bfloat16* vsrc = a.c.v;
                int bytes = 0;
                if (tok < cached) {
                    if (page >= 0) {
                        const long long off = row_in_pool(a.c, page, tok) + piece * 8;
                        ksrc += off; vsrc += off; bytes = 16;
                    }
                } else if (tok < n) {                        // the new token
                    ksrc = a.k_new + b * a.kn_seq + h * a.kn_head + piece * 8;
                    vsrc = a.v_new + b * a.vn_seq + h * a.vn_head + piece * 8;
                    bytes = 16;
                }
                const uint32_t dst = row * kRowBytes + ((piece ^ (row & 7)) << 4);
                cp_async16(ks + dst, ksrc, bytes);
                cp_async16(vs + dst, vsrc, bytes);
            }
            if (lane == 0) {
                const int bits = (p0 < 0 && base < cached ? 1 : 0) | (p1 < 0 && base + 8 < cached ? 2 : 0);
                bad[warp][stage] = bits;
                if (bits != 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
            }
            if (cached < n && pc.grp == 0 && cached >= base && cached < base + kTile) {      // append the new token
                const int page = cached < base + 8 ? p0 : p1;
                if (page >= 0) {
                    const long long off = row_in_pool(a.c, page, cached) + piece * 8;
                    if (row_hi == 0)
                        *reinterpret_cast<uint4*>(a.c.k + off) =
                            *reinterpret_cast<const uint4*>(a.k_new + b * a.kn_seq + h * a.kn_head + piece * 8);
                    else
                        *reinterpret_cast<uint4*>(a.c.v + off) =
                            *reinterpret_cast<const uint4*>(a.v_new + b * a.vn_seq + h * a.vn_head + piece * 8);
                    const long long at = slot_in_pool(a.c, page, cached);
                    if (lane == 0 && a.c.positions != nullptr)
                        a.c.positions[at] = a.new_positions != nullptr ? a.new_positions[b] : cached;
                    if (lane == 0 && a.c.mass != nullptr && !a.accumulate) a.c.mass[at] = 0.f;
                } else if (lane == 0 && a.status != nullptr) {
                    atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
                }
            }
            ++issued;
            if (++pc.tile == pc.tiles && issued < count) pc.next_unit(a);
        }
        cp_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) issue();

    // ---- consumer
    Cursor cc = start;
    const float scale2 = a.scale * kLog2e;
    const float cap_in = a.softcap > 0.f ? a.scale / a.softcap : 0.f, cap_out = a.softcap * kLog2e;
    uint32_t qf[NG][8][2];
    float o[NG][8][4];
    float mx[NG][2], sum[NG][2];
    bool fresh = true;
    int first_tile = 0, head0 = 0, heads = 0;

    for (int i = 0; i < count; ++i) {
        if (fresh) {                                         // a new unit or group: its queries
            fresh = false;
            first_tile = cc.tile;
            const int h = cc.unit / a.c.batch, b = cc.unit - h * a.c.batch;
            head0 = h * a.g + cc.grp * kDecodeHeads;
            heads = min(kDecodeHeads, a.g - cc.grp * kDecodeHeads);
            const __nv_bfloat16* q = a.q + b * a.q_seq;
#pragma unroll
            for (int t = 0; t < NG; ++t) {
                const bool live = t * 8 + gid < heads;
                const uint32_t* qh = reinterpret_cast<const uint32_t*>(q + (long long)(head0 + (live ? t * 8 + gid : 0)) * a.q_head);
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const uint32_t x0 = __ldg(qh + s * 8 + tig), x1 = __ldg(qh + s * 8 + tig + 4);
                    qf[t][s][0] = live ? x0 : 0u;
                    qf[t][s][1] = live ? x1 : 0u;
                    o[t][s][0] = o[t][s][1] = o[t][s][2] = o[t][s][3] = 0.f;
                }
                mx[t][0] = mx[t][1] = -INFINITY;
                sum[t][0] = sum[t][1] = 0.f;
            }
        }
        cp_wait<kStages - 1>();
        __syncwarp();
        const int stage = i % kStages;
        const uint32_t ks = ring_s + stage * kStageBytes, vs = ks + kTile * kRowBytes;
        const int base = cc.tile * kTile;

        // S^T: 16 tokens x 8 NG heads
        float s[NG][4];
#pragma unroll
        for (int t = 0; t < NG; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
        {
            const int row = (lane & 7) + ((lane >> 3) & 1) * 8, half = lane >> 4;
#pragma unroll
            for (int st = 0; st < 8; ++st) {
                uint32_t kf[4];
                ldsm4(kf, ks + row * kRowBytes + (((2 * st + half) ^ (row & 7)) << 4));
#pragma unroll
                for (int t = 0; t < NG; ++t) mma(s[t], kf, qf[t][st][0], qf[t][st][1]);
            }
        }
        // scores in base 2; what does not count gets -inf
        const int bits = bad[warp][stage];
        const int cached = cc.tokens - (a.k_new != nullptr);
        const int ta = base + gid, tb = ta + 8;
        const bool la = ta < cc.tokens && !((bits & 1) && ta < cached), lb = tb < cc.tokens && !((bits & 2) && tb < cached);
        uint32_t pf[NG][2];
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
                    pf[t][0] = transpose8x8(pack_bf16(__uint_as_float(pf[t][0]), pa));
                    pf[t][1] = transpose8x8(pack_bf16(__uint_as_float(pf[t][1]), pb));
                }
            }
        }
        if (a.accumulate) {                                  // kept until the sum over the whole unit is known
            float* row = a.scores + ((long long)(cc.before + cc.tile) * kTile + gid) * a.gs + cc.grp * kDecodeHeads + 2 * tig;
#pragma unroll
            for (int t = 0; t < NG; ++t)
                if (t * 8 + 2 * tig < heads) {
                    *reinterpret_cast<float2*>(row + t * 8) = make_float2(s[t][0], s[t][1]);
                    *reinterpret_cast<float2*>(row + t * 8 + 8 * (long long)a.gs) = make_float2(s[t][2], s[t][3]);
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
            const int row = (lane & 7) + (lane >> 4) * 8, half = (lane >> 3) & 1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t vf[4];
                ldsm4t(vf, vs + row * kRowBytes + (((2 * j + half) ^ (row & 7)) << 4));
#pragma unroll
                for (int t = 0; t < NG; ++t) mma(o[t][j], vf, pf[t][0], pf[t][1]);
            }
        }
        __syncwarp();
        issue();

        const bool unit_ends = ++cc.tile == cc.tiles;
        if (unit_ends || i + 1 == count) {                   // hand over what this warp has of the unit
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
            fresh = true;
            if (unit_ends && i + 1 < count) cc.next_unit(a);
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

// The pieces of a unit's group: partial slots [first, first + n).
struct Pieces { long long first; int n; };
__device__ __forceinline__ Pieces pieces_of(const DecodeArgs& a, int unit, int grp) {
    const int p = a.prefix[unit], tiles = a.prefix[unit + 1] - p;
    const long long total = (long long)a.prefix[a.units] * a.groups;
    const long long workers = min((long long)a.workers, total);
    const long long v = (long long)p * a.groups + (long long)grp * tiles;
    const int w0 = owner(v, total, workers), w1 = owner(v + tiles - 1, total, workers);
    return {(long long)w0 + (long long)unit * a.groups + grp, w1 - w0 + 1};
}

// Blocks [0, units * g): one (unit, query head) each; its pieces are joined: o = sum_i e_i o_i / sum_i e_i l_i with
// e_i = 2^(m_i - m).  The blocks behind them add the weights; each takes an equal run of tiles.
__global__ void __launch_bounds__(kThreads)
join_kernel(const __grid_constant__ DecodeArgs a, int join_blocks) {
    __shared__ float part[kWarps][kD];
    __shared__ float red_m[16][17], red_l[16][17];
    __shared__ float lse2[64];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    if ((int)blockIdx.x < join_blocks) {
        const int unit = blockIdx.x / a.g, head = blockIdx.x - unit * a.g;
        const int grp = head / kDecodeHeads, hh = head - grp * kDecodeHeads, gg = min(a.g, kDecodeHeads);
        const int h = unit / a.c.batch, b = unit - h * a.c.batch;
        __nv_bfloat16* dst = a.out + b * a.out_seq + (long long)(h * a.g + head) * a.out_head;
        float* lse = a.lse != nullptr ? a.lse + (long long)b * (a.c.heads * a.g) + h * a.g + head : nullptr;
        if (live_tokens(a, unit) == 0) {
            if (tid < kD) dst[tid] = __float2bfloat16_rn(0.f);
            if (tid == 0 && lse != nullptr) *lse = -INFINITY;
            return;
        }
        const Pieces ps = pieces_of(a, unit, grp);
        if (ps.n == 1) return;                               // written by the warp that had it whole
        float m = -INFINITY, l = 0.f;
        for (int i = lane; i < ps.n; i += 32) {
            const float* ml = a.ml + (ps.first + i) * 32 + hh;
            merge(m, l, ml[0], ml[16]);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const float mo = __shfl_xor_sync(0xffffffffu, m, d), lo = __shfl_xor_sync(0xffffffffu, l, d);
            merge(m, l, mo, lo);
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = warp; i < ps.n; i += kWarps) {
            const long long slot = ps.first + i;
            const float e = ex2f(a.ml[slot * 32 + hh] - ref);
            const float4 x = *reinterpret_cast<const float4*>(a.o + (slot * gg + hh) * kD + lane * 4);
            acc.x += e * x.x; acc.y += e * x.y; acc.z += e * x.z; acc.w += e * x.w;
        }
        *reinterpret_cast<float4*>(&part[warp][lane * 4]) = acc;
        __syncthreads();
        if (tid < kD) {
            float x = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) x += part[w][tid];
            dst[tid] = __float2bfloat16_rn(l == 0.f ? 0.f : x / l);
        }
        if (tid == 0 && lse != nullptr) *lse = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
        return;
    }

    // weights: w_j += sum over the unit's query heads of 2^(y_j - lse)
    const long long tiles = a.prefix[a.units];
    const int blk = blockIdx.x - join_blocks, blks = gridDim.x - join_blocks;
    long long t = blk * tiles / blks;
    const long long t1 = (blk + 1) * tiles / blks;
    if (t >= t1) return;
    int lo = 0, hi = a.units;                                // prefix[lo] <= t < prefix[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const bool below = at < hi && a.prefix[at] <= t;
        const int k = 31 - __clz(__ballot_sync(0xffffffffu, below));
        lo += k * step;
        hi = min(hi, lo + step);
    }
    int unit = lo;
    while (t < t1) {
        while (a.prefix[unit + 1] <= t) ++unit;              // units without tiles
        const int p = a.prefix[unit];
        const int tok0 = (int)(t - p) * kTile;
        const long long t_end = min(t1, (long long)a.prefix[unit + 1]);
        const int n = live_tokens(a, unit), tok1 = min(n, (int)(t_end - p) * kTile);
        const int cached = n - (a.k_new != nullptr);
        for (int grp = 0; grp < a.groups; ++grp) {
            const Pieces ps = pieces_of(a, unit, grp);
            const int heads = min(kDecodeHeads, a.g - grp * kDecodeHeads);
            const int hh = tid & 15, st = tid >> 4;
            float m = -INFINITY, l = 0.f;
            if (hh < heads)
                for (int i = st; i < ps.n; i += 16) {
                    const float* ml = a.ml + (ps.first + i) * 32 + hh;
                    merge(m, l, ml[0], ml[16]);
                }
            red_m[st][hh] = m; red_l[st][hh] = l;
            __syncthreads();
            if (tid < heads) {
                m = red_m[0][tid]; l = red_l[0][tid];
#pragma unroll
                for (int i = 1; i < 16; ++i) merge(m, l, red_m[i][tid], red_l[i][tid]);
                lse2[grp * kDecodeHeads + tid] = l == 0.f ? INFINITY : m + log2f(l);
            }
            __syncthreads();
        }
        for (int tok = tok0 + tid; tok < tok1; tok += kThreads) {
            const float2* row = reinterpret_cast<const float2*>(a.scores + ((long long)p * kTile + tok) * a.gs);
            float w = 0.f;
            for (int i = 0; i < a.g; i += 2) {
                const float2 y = row[i >> 1];
                w += ex2f(y.x - lse2[i]);
                if (i + 1 < a.g) w += ex2f(y.y - lse2[i + 1]);
            }
            const int page = page_of(a.c, unit, tok);
            if (page >= 0) {
                const long long at = slot_in_pool(a.c, page, tok);
                a.c.mass[at] = tok < cached ? a.c.mass[at] + w : w;
            }
        }
        __syncthreads();
        t = t_end;
    }
}

}  // namespace

cudaError_t launch_paged_attention(const DecodeArgs& a, int sm_count, cudaStream_t stream) {
    const int grid = a.workers / kWarps;
    auto kernel = a.g <= 8 ? decode_kernel<1> : decode_kernel<2>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
    if (e != cudaSuccess) return e;
    kernel<<<grid, kThreads, kSmemBytes, stream>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const int join_blocks = a.units * a.g;
    int mass_blocks = 0;
    if (a.accumulate) {
        const long long tokens = (long long)a.units * a.capacity;
        mass_blocks = (int)min(4LL * sm_count, (tokens + kThreads - 1) / kThreads);
    }
    e = launch_chained(kPdlOther, join_kernel, dim3(join_blocks + mass_blocks), dim3(kThreads), 0, stream, a, join_blocks);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace compactor
