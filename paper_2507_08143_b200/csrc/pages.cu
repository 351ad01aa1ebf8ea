// Choice of the pages that the queries of one new token per sequence attend to, out of the least and greatest key of every page.
//
//   score(page) = max over the KV head's query heads of sum_c (q_c > 0 ? q_c greatest_c : q_c least_c)
//
// is the most that q.k can be for a key between the bounds.  The first and the last pages of a unit are always taken, the other places
// go to the greatest scores (of equal ones the lower page).  What comes out is a row of a page table and a length, in the order of the
// unit's pages, so that the attention takes it like any other unit and the new token finds its slot behind the last one.
//
// The choice must not depend on the order of a sum, and next to the last place that is given away scores lie as close as they like; sums
// in 64 bits for all pages, though, took 15 us for 8 x 2048 pages and 34 for 128 ragged units, most of it conversions.  So there are two kernels:
//   1. scores by matrix instructions, 16 pages a warp: the sum is [least | greatest] times [min(q, 0) | max(q, 0)], products exact, sums in fp32; and a
//      bound of each score's error, from the same sum over absolute values.
//   2. a block per unit finds the T that the last place would go to by these scores.  With E the greatest of the error bounds, the last place's
//      true score lies within E of T, so a page more than 3 E above T is taken and one more than 3 E below is not, whatever the errors (and the one rounding
//      to fp32 that the definition has: 2^-24 of a score is far below E).  If there are just as many pages in between as places, all of them are taken;
//      else those few are summed again, in 64 bits and rounded once, and compared by that.
// Bound by the chain of launches and dependent reads (length, page ids, bounds, scores); the bytes are 512 per page.
#include "paged.cuh"
#include "quant4.cuh"

namespace compactor {
namespace {

constexpr uint32_t kKeyAlways = 0xffffffffu, kKeyNan = 0xfffffffeu;
constexpr int kScoreWarps = 4;
constexpr int kScorePages = 16 * kScoreWarps;

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

__global__ void __launch_bounds__(kScoreWarps * 32)
score_pages_kernel(const __grid_constant__ SelectArgs a, int chunks) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const long long t = select_tokens(a, unit);
    const int pages = t > 0 ? (int)((t + (1 << a.c.page_shift) - 1) >> a.c.page_shift) : 0;
    const int h = unit / a.c.batch, b = unit - h * a.c.batch;
    if (chunk == 0 && a.k_new != nullptr && t > 0 && warp == 0) {            // the new key enters the bounds of its page, whose score is not asked for
        const int page = page_of<false>(a.c, unit, (int)(t - 1)), piece = lane & 15;
        if (page >= 0) {
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
    }
    const int first = chunk * kScorePages + warp * 16;
    if (first >= pages || pages <= a.pages) return;          // (all pages are taken: no score is asked for)
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
        const int index = first + gid + 8 * p;
        if (tig == 0 && index < pages) {
            const bool always = index < a.first_pages || index >= pages - a.last_pages;
            const long long at = (long long)unit * a.unit_pages + index;
            a.keys[at] = always ? kKeyAlways : page[p] < 0 ? 0u : score_key(best[p]);
            a.errors[at] = always || page[p] < 0 ? 0.f : error[p];
        }
    }
}

// A block per unit: radix selection of the key of the last place (digits of 11, 11 and 10 bits), then the pages above it and, as far as there
// is room, the first of those that have it, in their order.
constexpr int kPickThreads = 512;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kBins = 2048;

struct PickShared {
    int hist[kBins];
    int warp_a[kPickWarps], warp_b[kPickWarps];
    float warp_e[kPickWarps];
    int digit, left;
};

// The count-th greatest of the keys; `left`: how many of the keys that equal it are among the count greatest.
__device__ __forceinline__ uint32_t last_place(PickShared& s, const uint32_t* key, int pages, int count, int& left) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kPer = kBins / kPickThreads;
    uint32_t prefix = 0;
    int shift = 32;
    left = count;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, next = shift - bits;
        *reinterpret_cast<int4*>(s.hist + tid * kPer) = make_int4(0, 0, 0, 0);
        static_assert(kPer == 4, "four bins a thread");
        __syncthreads();
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            if (pass == 0 || (k >> shift) == prefix) atomicAdd(&s.hist[(k >> next) & ((1u << bits) - 1u)], 1);
        }
        __syncthreads();
        // from the highest digit down: each thread a run of four
        const int4 v = *reinterpret_cast<const int4*>(s.hist + kBins - kPer - tid * kPer);
        const int c[4] = {v.w, v.z, v.y, v.x}, sum = v.x + v.y + v.z + v.w;
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) s.warp_a[warp] = upto;
        __syncthreads();
        int before = upto - sum;
#pragma unroll
        for (int w = 0; w < kPickWarps; ++w) before += w < warp ? s.warp_a[w] : 0;
        if (before < left && left <= before + sum) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < left && left <= before + c[i]) { s.digit = kBins - 1 - tid * kPer - i; s.left = left - before; }
                before += c[i];
            }
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint32_t)s.digit;
        left = s.left;
        shift = next;
    }
    return prefix;
}

// The score of a page as it is defined, summed in 64 bits and rounded once; by a warp, four channels a lane.
__device__ __forceinline__ uint32_t exact_key(const SelectArgs& a, int unit, int page) {
    const int lane = threadIdx.x & 31, h = unit / a.c.batch, b = unit - h * a.c.batch;
    const uint2 l = *(reinterpret_cast<const uint2*>(a.bounds + (long long)page * 2 * kD) + lane);
    const uint2 m = *(reinterpret_cast<const uint2*>(a.bounds + (long long)page * 2 * kD + kD) + lane);
    const float low[4] = {bf16_lo(l.x), bf16_hi(l.x), bf16_lo(l.y), bf16_hi(l.y)}, high[4] = {bf16_lo(m.x), bf16_hi(m.x), bf16_lo(m.y), bf16_hi(m.y)};
    double best = -INFINITY;
    bool nan = false;
#pragma unroll 4
    for (int j = 0; j < a.g; ++j) {
        const uint2 v = *(reinterpret_cast<const uint2*>(a.q + b * a.q_seq + (long long)(h * a.g + j) * a.q_head) + lane);
        const float q[4] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
        double x = 0.;
#pragma unroll
        for (int c = 0; c < 4; ++c) x = fma((double)q[c], (double)(q[c] > 0.f ? high[c] : low[c]), x);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        nan |= x != x;
        best = fmax(best, x);
    }
    return nan ? kKeyNan : score_key((float)best);
}

__global__ void __launch_bounds__(kPickThreads)
pick_pages_kernel(const __grid_constant__ SelectArgs a) {
    extern __shared__ __align__(16) uint32_t key[];
    __shared__ __align__(16) PickShared s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x;
    const long long t = select_tokens(a, unit);
    const int page_tokens = 1 << a.c.page_shift;
    const int pages = t > 0 ? (int)((t + page_tokens - 1) >> a.c.page_shift) : 0, count = min(pages, a.pages);
    const int* row = a.c.table + (long long)unit * a.c.max_pages;
    int* out = a.table_out + (long long)unit * a.pages;
    if (tid == 0) {
        int n = (int)max(t, -1LL);                           // -1 where there is no sequence, or none that fits
        if (t > 0) n = (int)(t - (long long)(pages - count) * page_tokens) - (a.k_new != nullptr);
        if (t == -1) n = a.lengths[unit];
        a.lengths_out[unit] = n;
        if (t == -2 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
    }
    for (int i = count + tid; i < a.pages; i += kPickThreads) out[i] = -1;
    if (pages <= a.pages) {
        for (int i = tid; i < pages; i += kPickThreads) {
            const int id = row[i];
            out[i] = id;
            if ((unsigned)id >= (unsigned)a.c.n_pages && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
        }
        return;
    }
    const uint32_t* keys = a.keys + (long long)unit * a.unit_pages;
    const float* errors = a.errors + (long long)unit * a.unit_pages;
    float worst = 0.f;
    bool vague = false;                                      // scores that say nothing: bounds or queries that are not finite, or sums near the end of the range
#pragma unroll 4
    for (int i = tid; i < pages; i += kPickThreads) {
        const float e = errors[i];
        key[i] = keys[i];
        if (e < INFINITY) worst = fmaxf(worst, e);
        else vague = true;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) worst = fmaxf(worst, __shfl_xor_sync(0xffffffffu, worst, d));
    if (lane == 0) s.warp_e[warp] = worst;
    const bool any_vague = __syncthreads_or(vague);
#pragma unroll
    for (int w = 0; w < kPickWarps; ++w) worst = fmaxf(worst, s.warp_e[w]);
    if (any_vague) {
        for (int i = warp; i < pages; i += kPickWarps) {
            if (errors[i] < INFINITY) continue;
            const uint32_t k = exact_key(a, unit, row[i]);   // (its page is one: those that are none have no error)
            if (lane == 0) key[i] = k;
        }
        __syncthreads();
    }
    int left;
    const uint32_t last = last_place(s, key, pages, count, left);
    uint32_t from = last, upto = last;                       // keys in between share the `left` last places
    if (last != 0u && last < kKeyNan && key_score(last) - key_score(last) == 0.f && worst > 0.f) {
        from = max(1u, score_key(key_score(last) - 3.f * worst));
        upto = score_key(key_score(last) + 3.f * worst);
        int above = 0, between = 0;
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            above += k > upto;
            between += k >= from && k <= upto;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) { above += __shfl_xor_sync(0xffffffffu, above, d); between += __shfl_xor_sync(0xffffffffu, between, d); }
        if (lane == 0) { s.warp_a[warp] = above; s.warp_b[warp] = between; }
        __syncthreads();
        above = between = 0;
#pragma unroll
        for (int w = 0; w < kPickWarps; ++w) { above += s.warp_a[w]; between += s.warp_b[w]; }
        left = count - above;
        if (between > left) {
            for (int i0 = warp * 32; i0 < pages; i0 += kPickThreads) {       // a warp sums those of 32 pages one after the other
                const uint32_t k = i0 + lane < pages ? key[i0 + lane] : 0u;
                uint32_t mine = k > upto ? kKeyAlways : 0u;
                for (uint32_t m = __ballot_sync(0xffffffffu, k >= from && k <= upto); m != 0u; m &= m - 1u) {
                    const int at = __ffs(m) - 1;
                    const uint32_t x = exact_key(a, unit, row[i0 + at]);
                    if (lane == at) mine = x;
                }
                if (i0 + lane < pages) key[i0 + lane] = mine;
            }
            __syncthreads();
            from = upto = last_place(s, key, pages, count, left);
        }
    }
    // ---- emission: keys above `upto`, and the first `left` from `from` on
    const int per = ((pages + 31) / 32 + kPickWarps - 1) / kPickWarps * 32;          // a run of whole words of 32 pages per warp
    const int p0 = min(pages, warp * per), p1 = min(pages, p0 + per);
    int above = 0, ties = 0;
    for (int i = p0; i < p1; i += 32) {
        const bool in = i + lane < p1;
        const uint32_t k = in ? key[i + lane] : 0u;
        above += __popc(__ballot_sync(0xffffffffu, in && k > upto));
        ties += __popc(__ballot_sync(0xffffffffu, in && k >= from && k <= upto));
    }
    __syncthreads();                                         // (the sums of the warps are read until here)
    if (lane == 0) { s.warp_a[warp] = above; s.warp_b[warp] = ties; }
    __syncthreads();
    int at = 0, tie = 0;
    for (int w = 0; w < warp; ++w) { at += s.warp_a[w]; tie += s.warp_b[w]; }
    at += min(tie, left);
    const uint32_t lower = (1u << lane) - 1u;
    for (int i = p0; i < p1; i += 32) {
        const bool in = i + lane < p1;
        const uint32_t k = in ? key[i + lane] : 0u;
        const bool same = in && k >= from && k <= upto;
        const uint32_t ms = __ballot_sync(0xffffffffu, same);
        const bool take = in && (k > upto || (same && tie + __popc(ms & lower) < left));
        const uint32_t mt = __ballot_sync(0xffffffffu, take);
        if (take) {
            const int id = row[i + lane];
            out[at + __popc(mt & lower)] = id;
            if ((unsigned)id >= (unsigned)a.c.n_pages && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
        }
        at += __popc(mt);
        tie += __popc(ms);
    }
}

}  // namespace

cudaError_t launch_paged_select(const SelectArgs& a, cudaStream_t stream) {
    const int chunks = (a.unit_pages + kScorePages - 1) / kScorePages;
    cudaError_t e;
    if ((e = launch_chained(kPdlOther, score_pages_kernel, dim3((unsigned)(a.units * chunks)), dim3(kScoreWarps * 32), 0, stream, a, chunks)) != cudaSuccess) return e;
    static std::atomic<unsigned long long> done;
    if ((e = allow_smem(pick_pages_kernel, kSelectMaxPages * (int)sizeof(uint32_t), done)) != cudaSuccess) return e;
    return launch_chained(kPdlOther, pick_pages_kernel, dim3((unsigned)a.units), dim3(kPickThreads), sizeof(uint32_t) * (size_t)a.unit_pages, stream, a);
}

}  // namespace compactor
