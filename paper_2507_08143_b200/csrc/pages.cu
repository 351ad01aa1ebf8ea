// Choice of the pages that the queries of one new token per sequence attend to, out of the least and greatest key of every page.
//
//   score(page) = max over the KV head's query heads of sum_c (q_c > 0 ? q_c greatest_c : q_c least_c)
//
// is the most that q.k can be for a key between the bounds.  (Of a page in 4 bits the bounds are rounded to the nearest bf16, and keys that were appended entered as
// given, up to half a step away from what is held: a key of such a page may lie that far outside.)  The first and the last pages of a unit are always taken, the other places
// go to the greatest scores (of equal ones the lower page).  What comes out is a row of a page table and a length, in the order of the
// unit's pages, so that the attention takes it like any other unit and the new token finds its slot behind the last one.
//
// The choice must not depend on the order of a sum, and next to the last place that is given away scores lie as close as they like; sums
// in 64 bits for all pages, though, took 15 us for 8 x 2048 pages and 34 for 128 ragged units, most of it conversions.  So there are two kernels:
//   1. scores by matrix instructions, 16 pages a warp: the sum is [least | greatest] times [min(q, 0) | max(q, 0)], products exact, sums in fp32; and a
//      bound of each score's error, from the same sum over absolute values.  The warps of a grid that fills the GPU share the pages of all units.
//   2. a block per unit finds an interval of scores that holds the last place, by a histogram of 2048 even steps between the least and the greatest
//      score, and another within a step while it holds many pages.  With E the greatest of the error bounds, a page more than 2 E and
//      a little above the interval is taken and one as far below is not, whatever the errors (the little is for the one rounding to fp32 that
//      the definition has: 2^-24 of a score, where E / 16 is 2^-20 of its absolute values).  The few pages in between are summed again, in 64 bits and rounded once, and compared by that.
// Bound by the chain of launches and dependent reads (length, page ids, bounds, scores); the bytes are 512 per page.  64 of 2048 pages for 8 units 12.9 us,
// 64 of up to 1025 for 128 ragged ones 15.5 (all sums in 64 bits: 19 and 44); the second kernel about 5, 2 more where sums are taken again.
#include "paged.cuh"
#include "quant4.cuh"

namespace compactor {
namespace {

constexpr uint32_t kKeyAlways = 0xffffffffu, kKeyNan = 0xfffffffeu;
constexpr int kScoreWarps = 4;

__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return kKeyNan;                              // as in the other selections: not a number ranks above +inf
    const uint32_t u = __float_as_uint(x + 0.f);             // -0 is 0
    return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_score(uint32_t k) { return __uint_as_float((k & 0x80000000u) != 0u ? k & 0x7fffffffu : ~k); }

// Tokens that a unit is going to attend to, the new one included; -1 for a row without a sequence, -2 for one that does not fit.
__device__ __forceinline__ long long select_tokens(const SelectArgs& a, int unit) {
    const int n = a.lengths[unit];
    if (n < 0) return -1;
    const long long t = (long long)n + (a.k_new != nullptr);
    return t > a.capacity ? -2 : t;
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Error of a score: sums of 16 instructions in four chains of four, each of which may drop a unit of 2^-23 of its partial sum for each of 17
// summands, three additions: 71 2^-23 of the sum of absolute values (which is itself no more than that far off).
constexpr float kScoreError = 0x1p-16f;
// The last place of an fp32 is never below 2^-149, which each of the 256 products and their sums may lose as well.  Where the rest of the error is not
// far above that, it is added, unless there is nothing to lose: all queries or all bounds are 0.
constexpr float kLeastError = 0x1p-139f;

// The new key enters the bounds of its page, by a warp.  (That page is taken without a score.)
__device__ __forceinline__ void enter_new_key(const SelectArgs& a, int unit, int lane) {
    const long long t = select_tokens(a, unit);
    if (a.k_new == nullptr || t <= 0) return;
    const int page = page_of<false>(a.c, unit, (int)(t - 1)), piece = lane & 15, h = unit / a.c.batch, b = unit - h * a.c.batch;
    if (page < 0) return;
    const uint4 x = *(reinterpret_cast<const uint4*>(a.k_new + b * a.kn_seq + h * a.kn_head) + piece);
    uint4* at = reinterpret_cast<uint4*>(a.bounds + (long long)page * 2 * kD + (lane >> 4) * kD) + piece;
    uint4 y = x;
    if (((t - 1) & ((1 << a.c.page_shift) - 1)) != 0) {
        const uint4 old = *at;
        y = lane < 16 ? make_uint4(min_nan2(old.x, x.x), min_nan2(old.y, x.y), min_nan2(old.z, x.z), min_nan2(old.w, x.w))
                      : make_uint4(max_nan2(old.x, x.x), max_nan2(old.y, x.y), max_nan2(old.z, x.z), max_nan2(old.w, x.w));
    }
    *at = y;
}

// Runs of 16 pages of a unit whose scores are asked for.
__device__ __forceinline__ int runs_of(const SelectArgs& a, int unit) {
    const long long t = select_tokens(a, unit);
    const int pages = t > 0 ? (int)((t + (1 << a.c.page_shift) - 1) >> a.c.page_shift) : 0;
    return pages <= a.pages ? 0 : (pages + 15) / 16;         // (where all pages are taken: none)
}

// Scores of one run, by a warp.  `cum`, `per`: runs before the units unit = i per, for i = 0, 1, ...
__device__ __forceinline__ void score_run(const SelectArgs& a, const int* cum, int per, int run, int lane) {
    const int gid = lane >> 2, tig = lane & 3;
    int lo = 0, hi = kScoreWarps * 32;                       // cum[lo] <= run < cum[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cum[mid] <= run) lo = mid; else hi = mid;
    }
    int unit = lo * per, nth = run - cum[lo];
    for (int n = runs_of(a, unit); nth >= n; n = runs_of(a, unit)) {
        nth -= n;
        if (++unit >= a.units) return;                       // (only if lengths change under the call, which its caller rules out)
    }
    const int pages = (int)((select_tokens(a, unit) + (1 << a.c.page_shift) - 1) >> a.c.page_shift), first = 16 * nth;
    const int h = unit / a.c.batch, b = unit - h * a.c.batch;
    // rows gid and gid + 8 of the warp's pages; the lane has the 16-byte pieces tig + 4 i of their least and greatest values
    uint4 low[2][4], high[2][4];
    int page[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int index = first + gid + 8 * p;
        page[p] = index < pages ? page_of<false>(a.c, unit, index << a.c.page_shift) : -1;
        const uint4* at = reinterpret_cast<const uint4*>(a.bounds + (long long)max(page[p], 0) * 2 * kD) + tig;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            low[p][i] = at[4 * i];
            high[p][i] = at[kD / 8 + 4 * i];
        }
    }
    float best[2] = {-INFINITY, -INFINITY}, error[2] = {0.f, 0.f};
    for (int head0 = 0; head0 < a.g; head0 += 8) {
        const uint4* q = reinterpret_cast<const uint4*>(a.q + b * a.q_seq + (long long)(h * a.g + min(head0 + gid, a.g - 1)) * a.q_head) + tig;
        float x[4][4] = {}, y[4][4] = {};                    // scores and sums of absolute values, four chains each
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = q[4 * i];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            const uint32_t l[2][4] = {{low[0][i].x, low[0][i].y, low[0][i].z, low[0][i].w}, {low[1][i].x, low[1][i].y, low[1][i].z, low[1][i].w}};
            const uint32_t m[2][4] = {{high[0][i].x, high[0][i].y, high[0][i].z, high[0][i].w}, {high[1][i].x, high[1][i].y, high[1][i].z, high[1][i].w}};
            constexpr uint32_t kAbs = 0x7fff7fffu;
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const uint32_t n0 = min_nan2(w[j], 0u), n1 = min_nan2(w[j + 1], 0u), p0 = max_nan2(w[j], 0u), p1 = max_nan2(w[j + 1], 0u);
                mma(x[i], l[0][j], l[1][j], l[0][j + 1], l[1][j + 1], n0, n1);
                mma(x[i], m[0][j], m[1][j], m[0][j + 1], m[1][j + 1], p0, p1);
                mma(y[i], l[0][j] & kAbs, l[1][j] & kAbs, l[0][j + 1] & kAbs, l[1][j + 1] & kAbs, n0 & kAbs, n1 & kAbs);
                mma(y[i], m[0][j] & kAbs, m[1][j] & kAbs, m[0][j + 1] & kAbs, m[1][j + 1] & kAbs, p0 & kAbs, p1 & kAbs);
            }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {                        // (columns behind the last head are the last head once more)
            const float sum = (x[0][c] + x[1][c]) + (x[2][c] + x[3][c]), size = (y[0][c] + y[1][c]) + (y[2][c] + y[3][c]);
            best[c >> 1] = fmaxf(best[c >> 1], sum);
            error[c >> 1] = size <= 0x1p100f ? fmaxf(error[c >> 1], size * kScoreError) : INFINITY;          // (not a number: infinite as well)
        }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
#pragma unroll
        for (int d = 1; d <= 2; d *= 2) {
            best[p] = fmaxf(best[p], __shfl_xor_sync(0xffffffffu, best[p], d));
            error[p] = fmaxf(error[p], __shfl_xor_sync(0xffffffffu, error[p], d));
        }
    }
    if (__any_sync(0xffffffffu, fminf(error[0], error[1]) < 0x1p-110f)) {
        uint32_t asked = 0u;                                 // not 0 where a query is not
        for (int head = gid; head < a.g; head += 8) {
            const uint4* q = reinterpret_cast<const uint4*>(a.q + b * a.q_seq + (long long)(h * a.g + head) * a.q_head) + tig;
#pragma unroll
            for (int i = 0; i < 4; ++i) asked |= (q[4 * i].x | q[4 * i].y | q[4 * i].z | q[4 * i].w) & 0x7fff7fffu;
        }
        const bool any = __any_sync(0xffffffffu, asked != 0u);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint32_t bits = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                bits |= low[p][i].x | low[p][i].y | low[p][i].z | low[p][i].w | high[p][i].x | high[p][i].y | high[p][i].z | high[p][i].w;
            bits |= __shfl_xor_sync(0xffffffffu, bits, 1);
            bits |= __shfl_xor_sync(0xffffffffu, bits, 2);
            if (any && (bits & 0x7fff7fffu) != 0u) error[p] += kLeastError;
        }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int index = first + gid + 8 * p;
        if (tig == 0 && index < pages) {
            const bool always = index < a.first_pages || index >= pages - a.last_pages;
            const long long at = (long long)unit * a.unit_pages + index;
            a.keys[at] = always ? kKeyAlways : page[p] < 0 ? 0u : score_key(best[p]);
            a.errors[at] = always || page[p] < 0 ? 0.f : error[p];
        }
    }
}

__global__ void __launch_bounds__(kScoreWarps * 32, 4)       // (128 registers a thread)
score_pages_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int kThreads = kScoreWarps * 32;
    __shared__ int cum[kThreads + 1];                        // runs before each thread's share of the units
    __shared__ int warp_sum[kScoreWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_trigger();
    pdl_wait();
    const int per = (a.units + kThreads - 1) / kThreads, u0 = min(a.units, tid * per), u1 = min(a.units, u0 + per);
    int mine = 0;
    for (int u = u0; u < u1; ++u) mine += runs_of(a, u);
    int incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kScoreWarps; ++w) incl += w < warp ? warp_sum[w] : 0;
    cum[tid + 1] = incl;
    if (tid == 0) cum[0] = 0;
    __syncthreads();
    const int all = cum[kThreads];
    for (int run = warp * gridDim.x + blockIdx.x; run < all; run += kScoreWarps * gridDim.x) score_run(a, cum, per, run, lane);
    for (int unit = warp * gridDim.x + blockIdx.x; unit < a.units; unit += kScoreWarps * gridDim.x) enter_new_key(a, unit, lane);
}
// A load that stays where it stands.
__device__ __forceinline__ int load_here(const int* p) {
    int x;
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(x) : "l"(p));
    return x;
}

constexpr int kPickThreads = 512;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kBins = 2048;
constexpr int kFew = 32;                       // pages in an interval that are not worth another histogram
constexpr int kRounds = 8;                     // most histograms

struct PickShared {
    int hist[kBins];
    int warp_a[kPickWarps], warp_b[kPickWarps];
    uint32_t warp_x[kPickWarps], warp_y[kPickWarps], warp_e[kPickWarps];
    int step, step_before, step_count, listed;
    int list[kPickThreads];                    // pages next to the last place
    uint32_t list_key[kPickThreads];
};

// The score of a page for the unit's query heads from `first` up to `end` as it is defined, summed in 64 bits and rounded once; by a warp, four channels
// a lane.
__device__ __forceinline__ uint32_t exact_key(const SelectArgs& a, int unit, int page, int first, int end) {
    const int lane = threadIdx.x & 31, h = unit / a.c.batch, b = unit - h * a.c.batch;
    const uint2 l = *(reinterpret_cast<const uint2*>(a.bounds + (long long)page * 2 * kD) + lane);
    const uint2 m = *(reinterpret_cast<const uint2*>(a.bounds + (long long)page * 2 * kD + kD) + lane);
    const float low[4] = {bf16_lo(l.x), bf16_hi(l.x), bf16_lo(l.y), bf16_hi(l.y)}, high[4] = {bf16_lo(m.x), bf16_hi(m.x), bf16_lo(m.y), bf16_hi(m.y)};
    uint32_t best = 0u;
    for (int j = first; j < end; ++j) {
        const uint2 v = *(reinterpret_cast<const uint2*>(a.q + b * a.q_seq + (long long)(h * a.g + j) * a.q_head) + lane);
        const float q[4] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
        double x = 0.;
#pragma unroll
        for (int c = 0; c < 4; ++c) x = fma((double)q[c], (double)(q[c] > 0.f ? high[c] : low[c]), x);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        best = max(best, score_key((float)x));               // (not a number above all)
    }
    return best;
}

// Sums of two counts over the block, in every thread.
__device__ __forceinline__ void block_sums(PickShared& s, int& x, int& y) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    x = __reduce_add_sync(0xffffffffu, x);
    y = __reduce_add_sync(0xffffffffu, y);
    __syncthreads();
    if (lane == 0) { s.warp_a[warp] = x; s.warp_b[warp] = y; }
    __syncthreads();
    x = __reduce_add_sync(0xffffffffu, lane < kPickWarps ? s.warp_a[lane] : 0);
    y = __reduce_add_sync(0xffffffffu, lane < kPickWarps ? s.warp_b[lane] : 0);
}
// The least of x and the greatest of y and e.
__device__ __forceinline__ void block_range(PickShared& s, uint32_t& x, uint32_t& y, uint32_t& e) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    x = __reduce_min_sync(0xffffffffu, x);
    y = __reduce_max_sync(0xffffffffu, y);
    e = __reduce_max_sync(0xffffffffu, e);
    __syncthreads();
    if (lane == 0) { s.warp_x[warp] = x; s.warp_y[warp] = y; s.warp_e[warp] = e; }
    __syncthreads();
    x = __reduce_min_sync(0xffffffffu, lane < kPickWarps ? s.warp_x[lane] : 0xffffffffu);
    y = __reduce_max_sync(0xffffffffu, lane < kPickWarps ? s.warp_y[lane] : 0u);
    e = __reduce_max_sync(0xffffffffu, lane < kPickWarps ? s.warp_e[lane] : 0u);
}

__global__ void __launch_bounds__(kPickThreads)
pick_pages_kernel(const __grid_constant__ SelectArgs a) {
    extern __shared__ __align__(16) uint32_t key[];
    __shared__ __align__(16) PickShared s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x;
    // what the first pages of a unit are about is asked for before its length is known
    constexpr int kAhead = 4;
    const uint32_t* keys = a.keys + (long long)unit * a.unit_pages;
    const float* errors = a.errors + (long long)unit * a.unit_pages;
    const int* row = a.c.table + (long long)unit * a.c.max_pages;
    const bool scored = a.unit_pages > a.pages;
    uint32_t key_ahead[kAhead];
    float error_ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const bool in = scored && tid + j * kPickThreads < a.unit_pages;
        key_ahead[j] = in ? keys[tid + j * kPickThreads] : 0u;
        error_ahead[j] = in ? errors[tid + j * kPickThreads] : 0.f;
    }
    const long long t = select_tokens(a, unit);
    const int page_tokens = 1 << a.c.page_shift;
    const int pages = t > 0 ? (int)((t + page_tokens - 1) >> a.c.page_shift) : 0, count = min(pages, a.pages);
    int* out = a.table_out + (long long)unit * a.pages;
    if (tid == 0) {
        int n = (int)max(t, -1LL);                           // -1 where there is no sequence, or none that fits
        if (t > 0) n = (int)(t - (long long)(pages - count) * page_tokens) - (a.k_new != nullptr);
        if (t == -1) n = a.lengths[unit];
        a.lengths_out[unit] = n;
        if (t == -2 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
    }
    if (!scored && warp == kPickWarps - 1) enter_new_key(a, unit, lane);     // (else the first kernel has done it)
    for (int i = count + tid; i < a.pages; i += kPickThreads) out[i] = -1;
    if (pages <= a.pages) {
        for (int i = tid; i < pages; i += kPickThreads) {
            const int id = row[i];
            out[i] = id;
            if ((unsigned)id >= (unsigned)a.c.n_pages && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
        }
        return;
    }
    // pages that this thread has in the emission: a run of whole words of 32 pages per warp; their ids are asked for now
    const int per_warp = ((pages + 31) / 32 + kPickWarps - 1) / kPickWarps * 32;
    const int p0 = min(pages, warp * per_warp), p1 = min(pages, p0 + per_warp);
    int id_ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) id_ahead[j] = load_here(row + min(p0 + 32 * j + lane, max(p1, 1) - 1));
    uint32_t worst_bits = 0u, low_key = 0xffffffffu, high_key = 0u;          // greatest error; least and greatest of the finite scores
    int above = 0, between = 0;                              // keys above the finite scores, finite scores
    bool vague = false;                                      // scores that say nothing: bounds or queries that are not finite, or sums near the end of the range
    const uint32_t kInfinite = score_key(INFINITY), kLeast = score_key(-INFINITY);
    auto scan = [&](uint32_t k) {
        above += k >= kInfinite;
        if (k < kInfinite && k > kLeast) { ++between; low_key = min(low_key, k); high_key = max(high_key, k); }
    };
    auto take_in = [&](int i, uint32_t k, float e) {
        key[i] = k;
        if (e < INFINITY) { worst_bits = max(worst_bits, __float_as_uint(e)); scan(k); }
        else vague = true;
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (tid + j * kPickThreads < pages) take_in(tid + j * kPickThreads, key_ahead[j], error_ahead[j]);
    for (int i = tid + kAhead * kPickThreads; i < pages; i += kPickThreads) take_in(i, keys[i], errors[i]);
    if (__syncthreads_or(vague)) {
        for (int i = warp; i < pages; i += kPickWarps) {
            if (errors[i] < INFINITY) continue;
            const uint32_t k = exact_key(a, unit, row[i], 0, a.g);   // (its page is one: those that are none have no error)
            if (lane == 0) { key[i] = k; scan(k); }
        }
    }
    block_range(s, low_key, high_key, worst_bits);
    block_sums(s, above, between);
    const float worst = __uint_as_float(worst_bits);
    // Keys above `upto` are taken, those below `from` are not, the `left` last places go to those in between: to the first of them where they
    // are all alike.  At first: what has no finite score on either side of what has.
    uint32_t from = low_key, upto = high_key;
    float low = key_score(low_key), high = key_score(high_key);
    auto count_keys = [&]() {
        above = between = 0;
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            above += k > upto;
            between += k >= from && k <= upto;
        }
        block_sums(s, above, between);
    };
    bool alike = false;
    if (count <= above || above + between < count) {         // the last place goes to a key that is no finite score: always taken, not a number, infinite or of no page
        alike = true;
        const uint32_t special[5] = {kKeyAlways, kKeyNan, score_key(INFINITY), score_key(-INFINITY), 0u};
        for (int i = 0; i < 5; ++i) {
            from = upto = special[i];
            count_keys();
            if (above < count && count <= above + between) break;
        }
    }
    // ---- smaller and smaller intervals of scores around the last place
    for (int round = 0; !alike && between > kFew && round < kRounds; ++round) {
        if (upto == from) { alike = worst == 0.f; break; }
        const float per = (float)kBins / (high - low);       // (0, infinite or not a number where the scores leave no room for steps)
        if (!(per > 0.f) || !(per < 0x1p120f)) break;
        for (int i = tid; i < kBins; i += kPickThreads) s.hist[i] = 0;
        __syncthreads();
        auto step_of = [&](uint32_t k) { return min(kBins - 1, (int)((key_score(k) - low) * per)); };      // rises with the score, ties with ties
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            if (k >= from && k <= upto) atomicAdd(&s.hist[step_of(k)], 1);
        }
        __syncthreads();
        // from the highest step down: each thread a run of four
        constexpr int kPer = kBins / kPickThreads;
        static_assert(kPer == 4, "four steps a thread");
        const int4 v = *reinterpret_cast<const int4*>(s.hist + kBins - kPer - tid * kPer);
        const int c[4] = {v.w, v.z, v.y, v.x}, sum = v.x + v.y + v.z + v.w;
        int incl = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += o;
        }
        if (lane == 31) s.warp_a[warp] = incl;
        __syncthreads();
        int before = above + incl - sum + __reduce_add_sync(0xffffffffu, lane < warp ? s.warp_a[lane] : 0);
        if (before < count && count <= before + sum) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < count && count <= before + c[i]) { s.step = kBins - 1 - tid * kPer - i; s.step_before = before; s.step_count = c[i]; }
                before += c[i];
            }
        }
        __syncthreads();
        // the step's own least and greatest key: the next interval
        const int step = s.step;
        uint32_t least = 0xffffffffu, most = 0u;
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            if (k >= from && k <= upto && step_of(k) == step) { least = min(least, k); most = max(most, k); }
        }
        uint32_t unused = 0u;
        block_range(s, least, most, unused);
        const bool narrower = least > from || most < upto;
        above = s.step_before; between = s.step_count;
        from = least; upto = most;
        low = key_score(from); high = key_score(upto);
        if (!narrower || high - low <= worst) break;
    }
    // ---- what the errors leave open is summed again
    if (!alike && worst > 0.f) {
        from = max(1u, score_key(low - 2.0625f * worst));
        upto = min(kKeyNan - 1u, score_key(high + 2.0625f * worst));
        count_keys();
    }
    int left = count - above;
    if (!alike && between > left) {
        if (tid == 0) s.listed = 0;
        __syncthreads();
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            if (k >= from && k <= upto) {
                const int at = atomicAdd(&s.listed, 1);
                if (at < kPickThreads) { s.list[at] = i; s.list_key[at] = 0u; }
            }
        }
        __syncthreads();
        const int listed = s.listed;
        if (listed <= kPickThreads) {                        // each of the few is ranked against the others: of equal ones the lower page comes first
            for (int j = warp; j < listed * a.g; j += kPickWarps) {          // (a query head of one of them at a time: the chain of a sum is long)
                const int which = j / a.g, head = j - which * a.g;
                const uint32_t k = exact_key(a, unit, row[s.list[which]], head, head + 1);
                if (lane == 0) atomicMax(&s.list_key[which], k);
            }
            __syncthreads();
            if (tid < listed) {
                const uint32_t k = s.list_key[tid];
                const int i = s.list[tid];
                int rank = 0;
                for (int j = 0; j < listed; ++j) rank += s.list_key[j] > k || (s.list_key[j] == k && s.list[j] < i);
                key[i] = rank < left ? kKeyAlways : 0u;
            }
            __syncthreads();
            // (all of the list that is taken is above `upto` now)
            from = 1u; upto = max(from, upto);
            left = 0;
        } else {                                             // many scores as good as equal: their 64-bit sums, digit by digit
            for (int i = warp; i < pages; i += kPickWarps) {
                const uint32_t k = key[i];
                uint32_t x = k > upto ? kKeyAlways : 0u;
                if (k >= from && k <= upto) x = exact_key(a, unit, row[i], 0, a.g);
                if (lane == 0) key[i] = x;
            }
            __syncthreads();
            uint32_t last = 0u;                              // the greatest key that at least `count` are not below
            for (int bit = 31; bit >= 0; --bit) {
                from = last | 1u << bit; upto = 0xffffffffu;
                count_keys();
                if (between >= count) last = from;
            }
            from = upto = last;
            count_keys();
            left = count - above;
        }
    }
    // ---- emission: keys above `upto`, and the first `left` from `from` on
    int taken = 0, ties = 0;
    for (int i = p0; i < p1; i += 32) {
        const bool in = i + lane < p1;
        const uint32_t k = in ? key[i + lane] : 0u;
        taken += __popc(__ballot_sync(0xffffffffu, in && k > upto));
        ties += __popc(__ballot_sync(0xffffffffu, in && k >= from && k <= upto));
    }
    __syncthreads();                                         // (the sums of the warps are read until here)
    if (lane == 0) { s.warp_a[warp] = taken; s.warp_b[warp] = ties; }
    __syncthreads();
    int at = __reduce_add_sync(0xffffffffu, lane < warp ? s.warp_a[lane] : 0), tie = __reduce_add_sync(0xffffffffu, lane < warp ? s.warp_b[lane] : 0);
    at += min(tie, left);
    const uint32_t lower = (1u << lane) - 1u;
    auto emit = [&](int i, int id) {                         // 32 pages from the i-th on
        const bool in = i + lane < p1;
        const uint32_t k = in ? key[i + lane] : 0u;
        const bool same = in && k >= from && k <= upto;
        const uint32_t ms = __ballot_sync(0xffffffffu, same);
        const bool take = in && (k > upto || (same && tie + __popc(ms & lower) < left));
        const uint32_t mt = __ballot_sync(0xffffffffu, take);
        if (take) {
            out[at + __popc(mt & lower)] = id;
            if ((unsigned)id >= (unsigned)a.c.n_pages && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
        }
        at += __popc(mt);
        tie += __popc(ms);
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (p0 + 32 * j < p1) emit(p0 + 32 * j, id_ahead[j]);
    for (int i = p0 + 32 * kAhead; i < p1; i += 32) emit(i, i + lane < p1 ? row[i + lane] : -1);
}

}  // namespace

cudaError_t launch_paged_select(const SelectArgs& a, int sm_count, cudaStream_t stream) {
    cudaError_t e;
    if (a.unit_pages > a.pages) {                            // (else all pages of every unit are taken)
        const long long runs = (long long)a.units * ((a.unit_pages + 15) / 16);
        const int blocks = (int)min((runs + kScoreWarps - 1) / kScoreWarps, 4LL * sm_count);
        if ((e = launch_chained(kPdlOther, score_pages_kernel, dim3(blocks), dim3(kScoreWarps * 32), 0, stream, a)) != cudaSuccess) return e;
    }
    static std::atomic<unsigned long long> done;
    if ((e = allow_smem(pick_pages_kernel, kSelectMaxPages * (int)sizeof(uint32_t), done)) != cudaSuccess) return e;
    return launch_chained(kPdlOther, pick_pages_kernel, dim3((unsigned)a.units), dim3(kPickThreads), sizeof(uint32_t) * (size_t)a.unit_pages, stream, a);
}

}  // namespace compactor
