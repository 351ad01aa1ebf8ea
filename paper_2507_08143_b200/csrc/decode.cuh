// Device code shared by the kernels that attend to one new token per sequence: instructions, and the sharing out of all tiles of a
// layer among the warps of a grid.
#pragma once
#include "paged.cuh"

namespace compactor {
namespace decode {

constexpr int kTile = kDecodeTile;
constexpr int kUnitCost = kDecodeUnitCost;
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
// Warps that share the work: fewer where each gets many tiles (see launch_paged_attention).
__device__ __forceinline__ int active_workers(const DecodeArgs& a, int total) {
    return total / 16 >= a.workers ? a.busy_workers : min(a.workers, total);
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

}  // namespace decode
}  // namespace compactor
