// Choice of the pages that the queries of one new token per sequence attend to, out of the least and greatest key of every page.
//
//   score(page) = max over the KV head's query heads of sum_c (q_c > 0 ? q_c greatest_c : q_c least_c)
//
// is the most that q.k can be for a key between the bounds.  The first and the last pages of a unit are always taken, the other places
// go to the greatest scores (of equal ones the lower page).  What comes out is a row of a page table and a length, in the order of the
// unit's pages, so that the attention takes it like any other unit and the new token finds its slot behind the last one.
//
// The sums are taken in 64 bits and rounded once: the choice must not depend on the order of a sum, and next to the last place that is
// given away scores lie as close as they like.  The bytes are few (512 per page), the multiply-adds 128 g per page at a 64th of the rate
// of a matrix instruction; two chained kernels, scores by blocks of 64 pages over the whole GPU, then a block per unit that selects.
#include "paged.cuh"
#include "quant4.cuh"

namespace compactor {
namespace {

constexpr uint32_t kKeyAlways = 0xffffffffu, kKeyNan = 0xfffffffeu;
constexpr int kScoreThreads = 256;
constexpr int kScorePages = 2 * kScoreThreads / 8;           // eight lanes have two pages

__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return kKeyNan;                              // as in the other selections: not a number ranks above +inf
    const uint32_t u = __float_as_uint(x + 0.f);             // -0 is 0
    return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}

// Tokens that a unit is going to attend to, the new one included; -1 for a row without a sequence, -2 for one that does not fit.
__device__ __forceinline__ long long select_tokens(const SelectArgs& a, int unit) {
    const int n = a.lengths[unit];
    if (n < 0) return -1;
    const long long t = (long long)n + (a.k_new != nullptr);
    return t > a.capacity ? -2 : t;
}

// HEADS query heads at a time: their sums for two pages are what a lane holds.
template <int HEADS>
__global__ void __launch_bounds__(kScoreThreads)
score_pages_kernel(const __grid_constant__ SelectArgs a, int chunks) {
    __shared__ double qs[HEADS][16][8];                      // [head][channel of the lane][lane of eight]: neighbouring lanes next to each other
    const int tid = threadIdx.x, sub = tid & 7, group = tid >> 3;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const long long t = select_tokens(a, unit);
    const int pages = t > 0 ? (int)((t + (1 << a.c.page_shift) - 1) >> a.c.page_shift) : 0;
    const int h = unit / a.c.batch, b = unit - h * a.c.batch;
    if (chunk == 0 && a.k_new != nullptr && t > 0 && tid < 32) {             // the new key enters the bounds of its page, whose score is not asked for
        const int page = page_of<false>(a.c, unit, (int)(t - 1)), piece = tid & 15;
        if (page >= 0) {
            const uint4 x = *(reinterpret_cast<const uint4*>(a.k_new + b * a.kn_seq + h * a.kn_head) + piece);
            uint4* at = reinterpret_cast<uint4*>(a.bounds + (long long)page * 2 * kD + (tid >> 4) * kD) + piece;
            uint4 y = x;
            if (((t - 1) & ((1 << a.c.page_shift) - 1)) != 0) {
                const uint4 old = *at;
                y = tid < 16 ? make_uint4(min_nan2(old.x, x.x), min_nan2(old.y, x.y), min_nan2(old.z, x.z), min_nan2(old.w, x.w))
                             : make_uint4(max_nan2(old.x, x.x), max_nan2(old.y, x.y), max_nan2(old.z, x.z), max_nan2(old.w, x.w));
            }
            *at = y;
        }
    }
    const int first = chunk * kScorePages;
    if (first >= pages || pages <= a.pages) return;          // (all pages are taken: no score is asked for)
    const int index[2] = {first + group, first + kScorePages / 2 + group};
    int page[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        page[p] = -1;
        if (index[p] < pages) page[p] = page_of<false>(a.c, unit, index[p] << a.c.page_shift);
    }
    uint4 least[2][2], most[2][2];                           // channels 8 sub + 0..7 and 64 + 8 sub + 0..7
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4* at = reinterpret_cast<const uint4*>(a.bounds + (long long)max(page[p], 0) * 2 * kD) + 8 * i + sub;
            least[p][i] = at[0];
            most[p][i] = at[kD / 8];
        }
    double best[2] = {-INFINITY, -INFINITY};
    bool nan[2] = {false, false};
    for (int head0 = 0; head0 < a.g; head0 += HEADS) {
        __syncthreads();
        for (int i = tid; i < HEADS * kD; i += kScoreThreads) {
            const int head = min(head0 + i / kD, a.g - 1), c = i % kD;       // (behind the last head: the last once more)
            qs[i / kD][(c >> 6) * 8 + (c & 7)][(c >> 3) & 7] = (double)__bfloat162float(a.q[b * a.q_seq + (long long)(h * a.g + head) * a.q_head + c]);
        }
        __syncthreads();
        double sum[2][HEADS];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int j = 0; j < HEADS; ++j) sum[p][j] = 0.;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lw[2][4] = {{least[0][i].x, least[0][i].y, least[0][i].z, least[0][i].w}, {least[1][i].x, least[1][i].y, least[1][i].z, least[1][i].w}};
            const uint32_t mw[2][4] = {{most[0][i].x, most[0][i].y, most[0][i].z, most[0][i].w}, {most[1][i].x, most[1][i].y, most[1][i].z, most[1][i].w}};
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                double lo[2], hi[2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    lo[p] = (double)((c & 1) != 0 ? bf16_hi(lw[p][c >> 1]) : bf16_lo(lw[p][c >> 1]));
                    hi[p] = (double)((c & 1) != 0 ? bf16_hi(mw[p][c >> 1]) : bf16_lo(mw[p][c >> 1]));
                }
#pragma unroll
                for (int j = 0; j < HEADS; ++j) {
                    const double q = qs[j][8 * i + c][sub];
#pragma unroll
                    for (int p = 0; p < 2; ++p) sum[p][j] = fma(q, q > 0. ? hi[p] : lo[p], sum[p][j]);
                }
            }
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int j = 0; j < HEADS; ++j) {
                double x = sum[p][j];
#pragma unroll
                for (int d = 1; d < 8; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
                nan[p] |= x != x;
                best[p] = fmax(best[p], x);
            }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
        if (sub == 0 && index[p] < pages) {
            const bool always = index[p] < a.first_pages || index[p] >= pages - a.last_pages;
            a.keys[(long long)unit * a.unit_pages + index[p]] =
                always ? kKeyAlways : page[p] < 0 ? 0u : nan[p] ? kKeyNan : score_key((float)best[p]);
        }
}

// A block per unit: radix selection of the key of the last place (digits of 11, 11 and 10 bits), then the pages above it and, as far as there
// is room, the first of those that have it, in their order.
constexpr int kPickThreads = 512;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kBins = 2048;

__global__ void __launch_bounds__(kPickThreads)
pick_pages_kernel(const __grid_constant__ SelectArgs a) {
    extern __shared__ __align__(16) uint32_t key[];
    __shared__ int hist[kBins];
    __shared__ int warp_sum[kPickWarps], warp_ties[kPickWarps];
    __shared__ int found_digit, found_left, found_in;
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
    for (int i = tid; i < pages; i += kPickThreads) key[i] = keys[i];
    // ---- the key of the last place: `left` of those that match `prefix` so far are taken, from the greatest on
    int left = count, shift = 32, in_bin = pages;
    uint32_t prefix = 0;
    for (int pass = 0; pass < 3 && left < in_bin; ++pass) {
        const int bits = pass < 2 ? 11 : 10, next = shift - bits;
        for (int i = tid; i < kBins; i += kPickThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < pages; i += kPickThreads) {
            const uint32_t k = key[i];
            if (pass == 0 || (k >> shift) == prefix) atomicAdd(&hist[(k >> next) & ((1u << bits) - 1u)], 1);
        }
        __syncthreads();
        // from the highest digit down: each thread a run of four
        int c[kBins / kPickThreads], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins / kPickThreads; ++i) {
            c[i] = hist[kBins - 1 - (tid * (kBins / kPickThreads) + i)];
            sum += c[i];
        }
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) warp_sum[warp] = upto;
        __syncthreads();
        int before = upto - sum;
#pragma unroll
        for (int w = 0; w < kPickWarps; ++w) before += w < warp ? warp_sum[w] : 0;
#pragma unroll
        for (int i = 0; i < kBins / kPickThreads; ++i) {
            if (before < left && left <= before + c[i]) {
                found_digit = kBins - 1 - (tid * (kBins / kPickThreads) + i);
                found_left = left - before;
                found_in = c[i];
            }
            before += c[i];
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint32_t)found_digit;
        left = found_left; in_bin = found_in;
        shift = next;
    }
    // ---- emission: keys above the prefix, and the first `left` that match it
    const uint32_t rest = shift == 0 ? 0u : (shift == 32 ? 0xffffffffu : (1u << shift) - 1u);
    const uint32_t first_match = shift == 32 ? 0u : prefix << shift, last_match = first_match | rest;
    const int per = ((pages + 31) / 32 + kPickWarps - 1) / kPickWarps * 32;          // a run of whole words of 32 pages per warp
    const int p0 = min(pages, warp * per), p1 = min(pages, p0 + per);
    int above = 0, ties = 0;
    for (int i = p0; i < p1; i += 32) {
        const bool in = i + lane < p1;
        const uint32_t k = in ? key[i + lane] : 0u;
        above += __popc(__ballot_sync(0xffffffffu, in && k > last_match));
        ties += __popc(__ballot_sync(0xffffffffu, in && k >= first_match && k <= last_match));
    }
    __syncthreads();                                         // (warp_sum is read until here)
    if (lane == 0) { warp_sum[warp] = above; warp_ties[warp] = ties; }
    __syncthreads();
    int at = 0, tie = 0;
    for (int w = 0; w < warp; ++w) { at += warp_sum[w]; tie += warp_ties[w]; }
    at += min(tie, left);
    const uint32_t lower = (1u << lane) - 1u;
    for (int i = p0; i < p1; i += 32) {
        const bool in = i + lane < p1;
        const uint32_t k = in ? key[i + lane] : 0u;
        const bool same = in && k >= first_match && k <= last_match;
        const uint32_t ms = __ballot_sync(0xffffffffu, same);
        const bool take = in && (k > last_match || (same && tie + __popc(ms & lower) < left));
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
    const auto score = a.g <= 2 ? score_pages_kernel<2> : a.g <= 4 ? score_pages_kernel<4> : score_pages_kernel<8>;
    if ((e = launch_chained(kPdlOther, score, dim3((unsigned)(a.units * chunks)), dim3(kScoreThreads), 0, stream, a, chunks)) != cudaSuccess) return e;
    static std::atomic<unsigned long long> done;
    if ((e = allow_smem(pick_pages_kernel, kSelectMaxPages * (int)sizeof(uint32_t), done)) != cudaSuccess) return e;
    return launch_chained(kPdlOther, pick_pages_kernel, dim3((unsigned)a.units), dim3(kPickThreads), sizeof(uint32_t) * (size_t)a.unit_pages, stream, a);
}

}  // namespace compactor
