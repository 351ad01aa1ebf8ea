// Rows out of the pages of a cache into dense tensors, the counterpart of the fill: token first[u] + j of a unit goes to row cu_seqlens[b] + j of
// its (layer, head).  Rows held in 4 bits come out as the bf16 nearest to lo + s c.
//
// Bound by HBM: 512 or 160 bytes read and 512 written per token (256 units x 2458 rows in 4 bits 69.7 us = 6.3 TB/s, 0.97 of the copy rate).  A block moves 128 rows: a thread per row finds its source (length and
// page id, two dependent reads), then 16 threads per row move 16 bytes of K and of V each, four rows of a thread in flight.
#include "paged.cuh"
#include "quant4.cuh"

namespace compactor {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;
constexpr int kRowsPerIter = kThreads / 16;
constexpr int kBatch = 4;

template <bool FOUR>
__global__ void __launch_bounds__(kThreads)
read_kernel(const __grid_constant__ ReadArgs a, const __grid_constant__ ReadTables t) {
    __shared__ long long src[kRows];                         // elements; < 0: the row is left alone
    const int tid = threadIdx.x;
    pdl_trigger();
    pdl_wait();
    const int layer = blockIdx.y / a.c.heads, head = blockIdx.y - layer * a.c.heads;
    const int row0 = t.cu_seqlens[0] + blockIdx.x * kRows, end = t.cu_seqlens[a.nb];
    if (tid < kRows) {
        long long from = -1;
        if (row0 + tid < end) {
            const int b = find_segment(t.cu_seqlens, a.nb, row0 + tid);
            const int unit = ((a.first_layer + layer) * a.c.heads + head) * a.c.batch + a.b0 + b;
            const int n = a.lengths[unit], first = a.first != nullptr ? a.first[unit] : 0;
            const long long token = (long long)first + row0 + tid - t.cu_seqlens[b];
            if (n > ((long long)a.c.max_pages << a.c.page_shift)) {
                if (a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
            } else if (first >= 0 && token < n) {
                const int page = page_of<false>(a.c, unit, (int)token);
                if (page >= 0) from = row_in_pool(a.c, page, (int)token);
                else if (a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
            }
        }
        src[tid] = from;
    }
    __syncthreads();
    const int piece = tid & 15, sub = tid >> 4, rows = min(kRows, end - row0);
    __nv_bfloat16* k = a.k + layer * a.k_layer + head * a.k_head + piece * 8;
    __nv_bfloat16* v = a.v + layer * a.v_layer + head * a.v_head + piece * 8;
#pragma unroll 1
    for (int r0 = sub; r0 < rows; r0 += kRowsPerIter * kBatch) {
        uint4 kv[kBatch], vv[kBatch];                        // (in 4 bits: a word of codes and the group's step and least value)
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const long long from = max(src[min(r0 + u * kRowsPerIter, rows - 1)], 0LL);
            if (FOUR) {
                const unsigned char* ks = reinterpret_cast<const unsigned char*>(a.c.k + from);
                const unsigned char* vs = reinterpret_cast<const unsigned char*>(a.c.v + from);
                kv[u].x = *reinterpret_cast<const uint32_t*>(ks + 4 * piece);
                kv[u].y = *reinterpret_cast<const uint32_t*>(ks + kRow4Codes + (piece & ~3));
                vv[u].x = *reinterpret_cast<const uint32_t*>(vs + 4 * piece);
                vv[u].y = *reinterpret_cast<const uint32_t*>(vs + kRow4Codes + (piece & ~3));
            } else {
                kv[u] = *(reinterpret_cast<const uint4*>(a.c.k + from) + piece);
                vv[u] = *(reinterpret_cast<const uint4*>(a.c.v + from) + piece);
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int r = r0 + u * kRowsPerIter;
            if (r >= rows || src[r] < 0) continue;
            *reinterpret_cast<uint4*>(k + (row0 + r) * a.k_token) = FOUR ? values8(kv[u].x, kv[u].y) : kv[u];
            *reinterpret_cast<uint4*>(v + (row0 + r) * a.v_token) = FOUR ? values8(vv[u].x, vv[u].y) : vv[u];
        }
    }
}

// ------------------------------------------------------------------------------------------ bounds
// Least and greatest key of a page, channel by channel, over its tokens: what the choice of pages goes by.  The least and greatest of a lane's
// channels stay packed, two to a register (min and max of bf16 are exact; they keep a not-a-number).  A warp takes a whole page where there are
// enough pages for all warps of the GPU, so that its chain of reads (length, page id, rows) is made once; up to eight share one where there are few.
constexpr int kBoundsThreads = 256;
constexpr int kBoundsWarps = kBoundsThreads / 32;

// Rows of bf16: 16 lanes hold a row, eight channels each, and 16 rows are in flight.  Bound by HBM, 256 bytes per token: 256 units x 2457 tokens on pages of
// 16 32.3 us = 5.6 TB/s, 0.86 of the copy rate.
struct Bounds16 {
    static constexpr int kRows = 16;                         // in flight
    static constexpr bool kAhead = false;                    // the next rows are asked for before these are looked at
    static constexpr int kBlocks = 5;                        // per SM
    struct Rows { uint4 x[8]; };
    uint32_t least[4], most[4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 4; ++i) { least[i] = 0x7f807f80u; most[i] = 0xff80ff80u; }
    }
    // rows [r0, r0 + kRows) of a page (behind the last of `tokens` the last once more)
    static __device__ __forceinline__ void fetch(Rows& r, const __nv_bfloat16* page, long long stride, int r0, int tokens, int lane) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.x[i] = *(reinterpret_cast<const uint4*>(page + min(r0 + 2 * i + (lane >> 4), tokens - 1) * stride) + (lane & 15));
    }
    __device__ __forceinline__ void take(const Rows& r) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w[4] = {r.x[i].x, r.x[i].y, r.x[i].z, r.x[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { least[j] = min_nan2(least[j], w[j]); most[j] = max_nan2(most[j], w[j]); }
        }
    }
    // over the lanes; then `words` are what the lane writes
    __device__ __forceinline__ void join(int lane, uint32_t (&words)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            least[j] = min_nan2(least[j], __shfl_xor_sync(0xffffffffu, least[j], 16));
            most[j] = max_nan2(most[j], __shfl_xor_sync(0xffffffffu, most[j], 16));
            words[j] = lane < 16 ? least[j] : most[j];
        }
    }
    static __device__ __forceinline__ uint32_t merge(int, uint32_t x, uint32_t y, int lane) { return lane < 16 ? min_nan2(x, y) : max_nan2(x, y); }
    static __device__ __forceinline__ void write(__nv_bfloat16* bounds, const uint32_t (&words)[4], int lane) {
        *(reinterpret_cast<uint4*>(bounds + (lane >> 4) * kD) + (lane & 15)) = make_uint4(words[0], words[1], words[2], words[3]);
    }
};

// Rows in 4 bits: a lane has a group of 32 channels of a row (16 bytes of codes, its step and least value), four lanes a row, 32 rows in flight.
// 80 bytes per token are few, so the instructions have to be: a code alone in the lower bits of a bf16 is c 2^-133, below the normal numbers
// (and one bit field up 16 c 2^-133, which runs on into the first normal ones), so that a mask and a product make numbers of two; the second product
// with s and the sum with lo are one more instruction, rounded once.  At the end eight lanes have the same channels: each round of the
// exchange halves what a lane keeps.  256 ragged units, 1.9 M tokens on pages of 64: 45.8 us = 3.6 TB/s, 0.56 of the copy rate, 64 % of the issue slots; with 16
// lanes a row and two instructions more per pair of channels 92.
struct Bounds4 {
    static constexpr int kRows = 32;
    static constexpr bool kAhead = true;                     // (61 -> 46 us for a ragged batch of 1.9 M tokens)
    static constexpr int kBlocks = 2;                        // (128 registers a thread; 8 bytes are spilled where many pages are gone through)
    struct Rows { uint4 codes[4]; uint32_t param[4]; };
    uint32_t least[16], most[16];                            // pair n of word j, channels 8 j + n and 8 j + n + 4 of the group, at 4 j + n
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 16; ++i) { least[i] = 0x7f807f80u; most[i] = 0xff80ff80u; }
    }
    static __device__ __forceinline__ void fetch(Rows& r, const __nv_bfloat16* page, long long, int r0, int tokens, int lane) {
        const unsigned char* rows = reinterpret_cast<const unsigned char*>(page);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned char* row = rows + min(r0 + 8 * i + (lane >> 2), tokens - 1) * kRow4;
            r.codes[i] = *reinterpret_cast<const uint4*>(row + 16 * (lane & 3));
            r.param[i] = *reinterpret_cast<const uint32_t*>(row + kRow4Codes + 4 * (lane & 3));
        }
    }
    __device__ __forceinline__ void take(const Rows& r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t s = __byte_perm(r.param[i], 0u, 0x1010), lo = __byte_perm(r.param[i], 0u, 0x3232);
            const uint32_t s0 = fma2(s, 0x43004300u, 0u), s1 = fma2(s, 0x41004100u, 0u);     // 2^7 s, 2^3 s
            const uint32_t w[4] = {r.codes[i].x, r.codes[i].y, r.codes[i].z, r.codes[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w8 = w[j] >> 8;
                const uint32_t c[4] = {w[j] & 0x000f000fu, w[j] & 0x00f000f0u, w8 & 0x000f000fu, w8 & 0x00f000f0u};
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t x = fma2(fma2(c[n], 0x7e807e80u, 0u), (n & 1) == 0 ? s0 : s1, lo);        // c 2^-133 * 2^126 * 2^7 s + lo
                    least[4 * j + n] = min_nan2(least[4 * j + n], x);
                    most[4 * j + n] = max_nan2(most[4 * j + n], x);
                }
            }
        }
    }
    // Lanes 2 KEEP apart exchange the pairs that they do not keep, KEEP of their 2 KEEP.
    template <int KEEP>
    __device__ __forceinline__ void halve(int lane) {
        const bool upper = (lane & (2 * KEEP)) != 0;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const uint32_t l = __shfl_xor_sync(0xffffffffu, upper ? least[i] : least[KEEP + i], 2 * KEEP);
            const uint32_t m = __shfl_xor_sync(0xffffffffu, upper ? most[i] : most[KEEP + i], 2 * KEEP);
            least[i] = min_nan2(upper ? least[KEEP + i] : least[i], l);
            most[i] = max_nan2(upper ? most[KEEP + i] : most[i], m);
        }
    }
    // The lane is left with two pairs: pairs n and n + 1 of word j (see write).
    __device__ __forceinline__ void join(int lane, uint32_t (&words)[4]) {
        halve<8>(lane);
        halve<4>(lane);
        halve<2>(lane);
        words[0] = least[0]; words[1] = least[1]; words[2] = most[0]; words[3] = most[1];
    }
    static __device__ __forceinline__ uint32_t merge(int i, uint32_t x, uint32_t y, int) { return i < 2 ? min_nan2(x, y) : max_nan2(x, y); }
    static __device__ __forceinline__ void write(__nv_bfloat16* bounds, const uint32_t (&words)[4], int lane) {
        const int j = (lane >> 4) * 2 + ((lane >> 3) & 1), n = ((lane >> 2) & 1) * 2;
        uint32_t* out = reinterpret_cast<uint32_t*>(bounds) + (32 * (lane & 3) + 8 * j + n) / 2;
        out[0] = __byte_perm(words[0], words[1], 0x5410);
        out[2] = __byte_perm(words[0], words[1], 0x7632);
        out[kD / 2] = __byte_perm(words[2], words[3], 0x5410);
        out[kD / 2 + 2] = __byte_perm(words[2], words[3], 0x7632);
    }
};

// Pages of a unit that are brought up to date: [first, end).
struct PageRange { int first, end, tokens; };
__device__ __forceinline__ PageRange pages_of(const BoundsArgs& a, int unit) {
    const int n = a.lengths[unit];
    if (n <= 0 || n > a.capacity) return {0, 0, 0};
    const int end = (int)(((long long)n + (1 << a.c.page_shift) - 1) >> a.c.page_shift);
    return {a.first != nullptr ? min(end, max(0, a.first[unit]) >> a.c.page_shift) : 0, end, n};
}
__device__ __forceinline__ int tokens_of(const BoundsArgs& a, const PageRange& r, int page) {
    return (int)min((long long)1 << a.c.page_shift, r.tokens - ((long long)page << a.c.page_shift));
}

// Many pages: the warps of a grid that fills the GPU take equal runs of them, whichever units they fall into.  (A block for every eight pages that
// there could be spends most of its time on those that there are not: ragged units of up to 32768 tokens, a quarter of that on average, 78 us.)
template <typename B>
__global__ void __launch_bounds__(kBoundsThreads, B::kBlocks)
bounds_kernel(const __grid_constant__ BoundsArgs a) {
    __shared__ int cum[kBoundsThreads + 1];                  // pages before each thread's share of the units
    __shared__ int warp_sum[kBoundsWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_trigger();
    pdl_wait();
    const int per = (a.units + kBoundsThreads - 1) / kBoundsThreads, u0 = min(a.units, tid * per), u1 = min(a.units, u0 + per);
    int mine = 0;
    for (int u = u0; u < u1; ++u) {
        const PageRange r = pages_of(a, a.first_unit + u);
        mine += r.end - r.first;
        if (blockIdx.x == 0 && a.status != nullptr && a.lengths[a.first_unit + u] > a.capacity) atomicOr(a.status + a.first_unit + u, COMPACTOR_STATUS_CAPACITY);
    }
    int incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBoundsWarps; ++w) incl += w < warp ? warp_sum[w] : 0;
    cum[tid + 1] = incl;
    if (tid == 0) cum[0] = 0;
    __syncthreads();
    const int all = cum[kBoundsThreads], warps = gridDim.x * kBoundsWarps, worker = warp * gridDim.x + blockIdx.x;
    const int begin = (int)((long long)all * worker / warps), end = (int)((long long)all * (worker + 1) / warps);
    if (begin >= end) return;
    int lo = 0, hi = kBoundsThreads;                         // cum[lo] <= begin < cum[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cum[mid] <= begin) lo = mid; else hi = mid;
    }
    int unit = a.first_unit + lo * per, left = begin - cum[lo];
    PageRange r = pages_of(a, unit);
    const int last_unit = a.first_unit + a.units - 1;        // (searches end there even if lengths change under the call, which its caller rules out)
    while (left >= r.end - r.first && unit < last_unit) {
        left -= r.end - r.first;
        r = pages_of(a, ++unit);
    }
    if (left >= r.end - r.first) return;
    int index = r.first + left, ids_from = index;            // lane l has the ids of pages ids_from + l
    auto ids_at = [&](int i) { return i + lane < r.end ? page_of<false>(a.c, unit, (i + lane) << a.c.page_shift) : -1; };
    int ids = ids_at(index);
    // rows [r0, r0 + kRows) of a page; page = -1 behind the last
    struct Place { int page, tokens, r0; };
    int to_come = end - begin;
    auto next_page = [&]() {
        while (to_come > 0) {
            --to_come;
            if (index == r.end) {                            // the next unit that has pages
                do {
                    if (unit >= last_unit) return Place{-1, 0, 0};
                    r = pages_of(a, ++unit);
                } while (r.end == r.first);
                index = ids_from = r.first;
                ids = ids_at(index);
            } else if (index == ids_from + 32) {
                ids_from = index;
                ids = ids_at(index);
            }
            const int page = __shfl_sync(0xffffffffu, ids, index - ids_from), tokens = tokens_of(a, r, index);
            ++index;
            if (page >= 0) return Place{page, tokens, 0};
            if (lane == 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
        }
        return Place{-1, 0, 0};
    };
    auto fetch = [&](typename B::Rows& rows, const Place& p) { B::fetch(rows, a.c.k + row_in_pool(a.c, p.page, 0), a.c.stride_token, p.r0, p.tokens, lane); };
    B acc;
    acc.clear();
    typename B::Rows rows, ahead;
    Place now = next_page();
    if (B::kAhead && now.page >= 0) fetch(ahead, now);
    while (now.page >= 0) {
        const bool page_ends = now.r0 + B::kRows >= now.tokens;
        const Place next = page_ends ? next_page() : Place{now.page, now.tokens, now.r0 + B::kRows};
        if (B::kAhead) {
            rows = ahead;
            if (next.page >= 0) fetch(ahead, next);
        } else {
            fetch(rows, now);
        }
        acc.take(rows);
        if (page_ends) {
            uint32_t words[4];
            acc.join(lane, words);
            B::write(a.bounds + (long long)now.page * 2 * kD, words, lane);
            acc.clear();
        }
        now = next;
    }
}

// Few pages: several warps share one.
template <typename B>
__global__ void __launch_bounds__(kBoundsThreads)
bounds_few_kernel(const __grid_constant__ BoundsArgs a, int chunks, int warps_per_page) {
    __shared__ uint32_t part[kBoundsWarps][4][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, way = warp % warps_per_page;
    pdl_trigger();
    pdl_wait();
    const int unit = a.first_unit + blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const int index = chunk * (kBoundsWarps / warps_per_page) + warp / warps_per_page;               // of the unit's pages
    const PageRange r = pages_of(a, unit);
    if (threadIdx.x == 0 && chunk == 0 && a.status != nullptr && a.lengths[unit] > a.capacity) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
    int page = -1;
    B acc;
    acc.clear();
    if (index >= r.first && index < r.end) {
        page = page_of<false>(a.c, unit, index << a.c.page_shift);
        if (page < 0 && lane == 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
    }
    if (page >= 0) {
        const int tokens = tokens_of(a, r, index);
        const __nv_bfloat16* rows = a.c.k + row_in_pool(a.c, page, 0);
#pragma unroll 1
        for (int r0 = B::kRows * way; r0 < tokens; r0 += B::kRows * warps_per_page) {
            typename B::Rows x;
            B::fetch(x, rows, a.c.stride_token, r0, tokens, lane);
            acc.take(x);
        }
    }
    uint32_t words[4];
    acc.join(lane, words);
#pragma unroll
    for (int i = 0; i < 4; ++i) part[warp][i][lane] = words[i];
    __syncthreads();
    if (way != 0 || page < 0) return;
    for (int o = 1; o < warps_per_page; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i) words[i] = B::merge(i, words[i], part[warp + o][i][lane], lane);
    B::write(a.bounds + (long long)page * 2 * kD, words, lane);
}

}  // namespace

cudaError_t launch_paged_read(const ReadArgs& a, const ReadTables& t, cudaStream_t stream) {
    const int rows = t.cu_seqlens[a.nb] - t.cu_seqlens[0];
    if (rows == 0) return cudaSuccess;
    const dim3 grid((unsigned)((rows + kRows - 1) / kRows), a.layers * a.c.heads);
    return launch_chained(kPdlOther, a.four ? read_kernel<true> : read_kernel<false>, grid, dim3(kThreads), 0, stream, a, t);
}

cudaError_t launch_paged_bounds(const BoundsArgs& a, int sm_count, cudaStream_t stream) {
    const int page = 1 << a.c.page_shift, pages = (a.capacity + page - 1) / page;
    int warps_per_page = 1;                                  // while there are not some warps for every SM's schedulers
    while (warps_per_page < kBoundsWarps && page > (a.four ? Bounds4::kRows : Bounds16::kRows) * warps_per_page &&
           (long long)a.units * pages * warps_per_page < 64LL * sm_count) warps_per_page *= 2;
    if (warps_per_page > 1) {
        const int per_block = kBoundsWarps / warps_per_page, chunks = (pages + per_block - 1) / per_block;
        return launch_chained(kPdlOther, a.four ? bounds_few_kernel<Bounds4> : bounds_few_kernel<Bounds16>, dim3((unsigned)(a.units * chunks)),
                              dim3(kBoundsThreads), 0, stream, a, chunks, warps_per_page);
    }
    const int blocks = (int)min(((long long)a.units * pages + kBoundsWarps - 1) / kBoundsWarps, (long long)(a.four ? Bounds4::kBlocks : Bounds16::kBlocks) * sm_count);
    return launch_chained(kPdlOther, a.four ? bounds_kernel<Bounds4> : bounds_kernel<Bounds16>, dim3((unsigned)blocks), dim3(kBoundsThreads), 0, stream, a);
}

}  // namespace compactor
