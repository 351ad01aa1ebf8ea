// The paged cache's two copying operators: filling pages with the rows that a selection kept, and evicting the tokens of
// least accumulated attention weight.  Both move whole 256-byte rows as 16-byte pieces, bit for bit.
#include "paged.cuh"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace compactor {
namespace {

// ------------------------------------------------------------------------------------------ fill
// Where a row goes: slot lengths[unit] + j of its unit, j its place among the unit's kept rows, found through the page table.  A block
// moves 128 rows: first a thread per row finds source and target (index, length and page id are three dependent reads,
// made once per row and not once per 16-byte piece) and moves weight and position, then 16 threads per row move K and V.
// Bound by HBM: 512 bytes read and written per row.  256 units x 2458 of 8192 rows: 109 us = 6.0 TB/s, 0.92 of the copy rate.
constexpr int kFillThreads = 256;
constexpr int kFillRows = 128;
constexpr int kFillRowsPerIter = kFillThreads / 16;
constexpr int kFillBatch = 4;                   // rows per thread in flight (2: 112.6 us instead of 111.0 for 32 x 8 heads x 2458 rows)

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Where the kept rows of unit (layer, head, sequence b) begin in idx, and how many there are.
__device__ __forceinline__ int kept_rows(const FillArgs& a, const FillTables& t, int layer, int head, int b) {
    if (a.head_offsets == nullptr) return t.cu_keep[b + 1] - t.cu_keep[b];
    const int* offs = a.head_offsets + ((long long)layer * a.c.batch + a.b0 + b) * (a.c.heads + 1);
    return max(0, offs[head + 1] - offs[head]);
}
// Slot of a unit's first new row; -1 if the unit takes none (no sequence in the row, or no room).
__device__ __forceinline__ int first_slot(const FillArgs& a, int unit, int rows) {
    const int n = a.lengths != nullptr ? a.lengths[unit] : 0;
    if (n < 0) return -1;
    return (long long)n + rows > ((long long)a.c.max_pages << a.c.page_shift) ? -1 : n;
}

// New lengths, and the units that had no room.
__device__ __forceinline__ void write_lengths(const FillArgs& a, const FillTables& t, long long i) {
    if (i >= (long long)a.layers * a.c.heads * a.nb) return;
    const int b = (int)(i % a.nb), lh = (int)(i / a.nb), layer = lh / a.c.heads, head = lh - layer * a.c.heads;
    const int unit = ((a.first_layer + layer) * a.c.heads + head) * a.c.batch + a.b0 + b;
    const int rows = kept_rows(a, t, layer, head, b), first = first_slot(a, unit, rows);
    const int n = a.lengths != nullptr ? a.lengths[unit] : 0;
    if (first < 0 && n >= 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
    if (a.lengths_out != nullptr) a.lengths_out[unit] = first < 0 ? n : n + rows;
}
// Where lengths_out is lengths, which every block of the fill reads, they are written by a launch of their own.
__global__ void fill_lengths_kernel(const __grid_constant__ FillArgs a, const __grid_constant__ FillTables t) {
    pdl_trigger();
    pdl_wait();
    write_lengths(a, t, (long long)blockIdx.x * blockDim.x + threadIdx.x);
}

template <bool ACROSS>
__global__ void __launch_bounds__(kFillThreads)
fill_kernel(const __grid_constant__ FillArgs a, const __grid_constant__ FillTables t, int row_blocks) {
    __shared__ long long src_k[kFillRows], src_v[kFillRows], dst[kFillRows];       // elements; dst < 0: the row is skipped
    const int tid = threadIdx.x;
    pdl_trigger();
    pdl_wait();
    if ((int)blockIdx.x >= row_blocks) {                     // blocks behind those with rows: the lengths, a row of the grid's share each
        const long long per = ((long long)a.layers * a.c.heads * a.nb + gridDim.y - 1) / gridDim.y;
        for (long long i = tid; i < per; i += kFillThreads) write_lengths(a, t, blockIdx.y * per + i);
        return;
    }
    const int layer = ACROSS ? blockIdx.y : blockIdx.y / a.c.heads;
    const long long per_outer = ACROSS ? (long long)a.c.heads * a.total_keep : a.total_keep;     // rows per layer or (layer, head)
    const int scale = ACROSS ? a.c.heads : 1;
    const long long end = (long long)scale * t.cu_keep[a.nb];
    const long long row0 = (long long)scale * t.cu_keep[0] + (long long)blockIdx.x * kFillRows;
    if (tid < kFillRows) {
        const long long row = row0 + tid;
        long long to = -1;
        if (row < end) {
            const int local0 = a.idx != nullptr ? a.idx[(long long)blockIdx.y * per_outer + row] : 0;
            const int b = find_segment(t.cu_keep, a.nb, (int)(row / scale));
            int head, j;
            if (ACROSS) {
                const int* offs = a.head_offsets + ((long long)layer * a.c.batch + a.b0 + b) * (a.c.heads + 1);
                j = (int)(row - (long long)scale * t.cu_keep[b]);
                head = find_segment(offs, a.c.heads, j);
                j -= offs[head];
            } else {
                head = blockIdx.y - layer * a.c.heads;
                j = (int)row - t.cu_keep[b];
            }
            const int n = t.cu_seqlens[b + 1] - t.cu_seqlens[b];
            const int local = a.idx != nullptr ? local0 : j;
            const int unit = ((a.first_layer + layer) * a.c.heads + head) * a.c.batch + a.b0 + b;
            const int rows = kept_rows(a, t, layer, head, b), first = first_slot(a, unit, rows);
            if (first >= 0 && j >= 0 && j < rows && (unsigned)local < (unsigned)n) {
                const int slot = first + j, page = page_of<false>(a.c, unit, slot);
                if (page >= 0) {
                    const long long tok = (long long)t.cu_seqlens[b] + local;
                    to = row_in_pool(a.c, page, slot);
                    src_k[tid] = layer * a.k.stride_layer + head * a.k.stride_head + tok * a.k.stride_token;
                    src_v[tid] = layer * a.v.stride_layer + head * a.v.stride_head + tok * a.v.stride_token;
                    const long long at = slot_in_pool(a.c, page, slot);
                    if (a.c.mass != nullptr)
                        a.c.mass[at] = a.mass_in != nullptr ? a.mass_in[((long long)layer * a.c.heads + head) * a.total_tokens + tok] : 0.f;
                    if (a.c.positions != nullptr)
                        a.c.positions[at] = (a.first_position != nullptr ? a.first_position[a.b0 + b] : 0) + local;
                } else if (a.status != nullptr) {
                    atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
                }
            }
        }
        dst[tid] = to;
        if (to < 0) src_k[tid] = src_v[tid] = 0;             // read, not written: any address of the tensor will do
    }
    __syncthreads();
    const int piece = tid & 15, sub = tid >> 4;
    const int rows_here = (int)min((long long)kFillRows, end - row0);
#pragma unroll 1
    for (int r0 = sub; r0 < rows_here; r0 += kFillRowsPerIter * kFillBatch) {
        uint4 kv[kFillBatch], vv[kFillBatch];
#pragma unroll
        for (int u = 0; u < kFillBatch; ++u) {               // without a condition, so that they are in flight together
            const int r = min(r0 + u * kFillRowsPerIter, rows_here - 1);
            kv[u] = ld_stream(reinterpret_cast<const uint4*>(a.k.ptr + src_k[r]) + piece);
            vv[u] = ld_stream(reinterpret_cast<const uint4*>(a.v.ptr + src_v[r]) + piece);
        }
#pragma unroll
        for (int u = 0; u < kFillBatch; ++u) {
            const int r = r0 + u * kFillRowsPerIter;
            if (r >= rows_here || dst[r] < 0) continue;
            *(reinterpret_cast<uint4*>(a.c.k + dst[r]) + piece) = kv[u];
            *(reinterpret_cast<uint4*>(a.c.v + dst[r]) + piece) = vv[u];
        }
    }
}

// ------------------------------------------------------------------------------------------ evict
// One CTA per unit, or a cluster (of up to 8, for few units up to 16), of which as many CTAs work as the unit's length asks for;
// each holds the sort keys of a slice of the unit's slots in shared memory.
//   key      the weight as an ordered 32-bit integer; the largest key for a recent token (never below a weight)
//   1. radix selection of the E-th smallest key, E = n - budget: digits of 11, 11 and 10 bits, one histogram per CTA,
//      summed over the cluster through distributed shared memory by every CTA alike; it ends as soon as all keys of the digit go
//   2. a bit per slot: evicted or not (of equal keys the higher slots go first)
//   3. lists of the holes (evicted, below the budget) and the movers (kept, at or above it), both ascending; there are as
//      many of one as of the other, and the j-th mover's row goes to the j-th hole.  Sources and targets never overlap, so the
//      rows move in any order, and no more than min(E, budget) of them move: compaction that kept the slots' order
//      would rewrite nearly the whole unit for one evicted token.
// The bytes are few (8 per slot, 1 KB per moved row); what bounds it is the chain of block-wide steps, about 8 us per unit
// whatever its length.  So several small CTAs share an SM and hide each other's waits.  One token out of each of 256 units of 2459:
// 8.6 us; 128 out of 512 ragged units of 9 K on average: 49 us; 8192 out of 8 units of 50136: 35 us.
constexpr int kBins = 2048;
constexpr int kMaxCluster = 16;                 // 8 is what every launch may use
constexpr int kSmallThreads = 256, kLargeThreads = 512;
// Most slots per CTA: 33 KB of keys, four CTAs to an SM; 192 KB, one.  The smaller is 8192 and a little more, so that a budget that is a power of
// two and a block of a few hundred tokens behind it need clusters of the budget's size (512 ragged units of up to 32896 tokens, 128 of them
// new: 49 us, with slices of 8192 53, of 9216 49).
constexpr int kSmallSlice = 8256, kLargeSlice = 49152;
constexpr int kLoadBatch = 8;                   // groups of four slots per thread whose weights are in flight together
constexpr uint32_t kKeyRecent = 0xffffffffu, kKeyNan = 0xfffffffeu;

template <int kThreads>
struct EvictShared {
    static constexpr int kWords = (kThreads == kSmallThreads ? kSmallSlice : kLargeSlice) / 32;
    int hist[2][kBins];                         // passes take turns
    int coarse[2][kBins / 32];
    uint32_t evicted[kWords];                   // bit per slot of the slice
    uint32_t same[kWords];                      // bit per slot whose key cannot be told from the E-th smallest
    int warp_a[kThreads / 32], warp_b[kThreads / 32];
    int holes, movers, ties, bad;               // of this CTA's slice
    int rank_holes[kMaxCluster], rank_movers[kMaxCluster];
    int digit, left, in_bin;
};

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return kKeyNan;                 // as in the selection of the prefill: not a number ranks above +inf
    const uint32_t u = __float_as_uint(w + 0.f);             // -0 is 0
    return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}

// Exclusive prefix over the block of two counts per thread, and their totals.
template <int kThreads>
__device__ __forceinline__ void block_prefix2(EvictShared<kThreads>& s, int& x, int& y, int& total_x, int& total_y) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int ix = x, iy = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int ox = __shfl_up_sync(0xffffffffu, ix, d), oy = __shfl_up_sync(0xffffffffu, iy, d);
        if (lane >= d) { ix += ox; iy += oy; }
    }
    __syncthreads();
    if (lane == 31) { s.warp_a[warp] = ix; s.warp_b[warp] = iy; }
    __syncthreads();
    int bx = 0, by = 0;
    total_x = total_y = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        const int cx = s.warp_a[w], cy = s.warp_b[w];
        if (w < warp) { bx += cx; by += cy; }
        total_x += cx; total_y += cy;
    }
    x = bx + ix - x; y = by + iy - y;
}

// One unit.  `part`: which units the launch is for.
enum { kEvictAll, kEvictLong, kEvictShort };
template <int kThreads, bool L2>
__device__ __forceinline__ void evict_unit(const EvictArgs& a, int slice_cap, int part) {
    constexpr int kWarps = kThreads / 32;
    constexpr int kRowBatch = kThreads == kSmallThreads ? 4 : 8;     // rows per warp in flight
    extern __shared__ __align__(16) uint32_t key[];          // [slice_cap]; afterwards the two lists
    __shared__ __align__(16) EvictShared<kThreads> s;
    int4* move = reinterpret_cast<int4*>(s.hist[0]);         // a batch of moves, when the histograms are done with: page and slot from, page and slot to
    cg::cluster_group cluster = cg::this_cluster();
    const int cluster_size = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int unit = a.first_unit + (int)(blockIdx.x / cluster_size);
    const int n = load<L2>(a.lengths + unit), budget = load<L2>(a.budgets + unit);
    const long long capacity = min((long long)a.max_length, (long long)a.c.max_pages << a.c.page_shift);
    if (part == kEvictLong ? n <= kSmallSlice : part == kEvictShort && n > kSmallSlice) return;
    // nothing to do: the same decision in every CTA of the cluster, before any barrier between them
    if (n < 0 || budget < 0 || n <= budget || n > capacity || budget == 0) {
        if (rank == 0 && tid == 0) {
            const bool refused = n > capacity;
            if (refused && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
            a.lengths_out[unit] = !refused && budget == 0 && n > 0 ? 0 : n;
        }
        return;
    }
    int ranks = 1;                                           // CTAs that this unit needs; a barrier of the cluster waits for those that have not ended
    while (ranks * slice_cap < n) ++ranks;
    if (rank >= ranks) return;
    auto sync_ranks = [&]() {
        if (ranks == 1) __syncthreads();
        else cluster.sync();
    };
    const int slice = ((n + ranks - 1) / ranks + 31) / 32 * 32;              // at most slice_cap
    const int lo = min(n, rank * slice), count = min(n, lo + slice) - lo;
    const int recent_from = a.recent > 0 ? (int)max((long long)load<L2>(a.next_position + unit % a.c.batch) - min(a.recent, budget), -0x80000000LL) : 0;

    if (tid == 0) s.bad = 0;
    for (int i = tid; i < 2 * kBins / 4; i += kThreads) reinterpret_cast<int4*>(s.hist)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    const uint32_t key_s = (uint32_t)__cvta_generic_to_shared(key);
    const int quads = (count + 3) / 4;                       // four slots share a page: one id, one 16-byte load of each pool
    for (int q0 = tid; q0 < quads; q0 += kThreads * kLoadBatch) {
        int page[kLoadBatch];
        int4 pos[kLoadBatch];
#pragma unroll
        for (int k = 0; k < kLoadBatch; ++k) page[k] = page_of<L2>(a.c, unit, lo + 4 * min(q0 + k * kThreads, quads - 1));
#pragma unroll
        for (int k = 0; k < kLoadBatch; ++k) {               // weights into the keys' place, positions into registers: all in flight at once
            const int q = min(q0 + k * kThreads, quads - 1);
            const long long at = slot_in_pool(a.c, max(page[k], 0), lo + 4 * q);
            if (q0 + k * kThreads < quads)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(key_s + 16 * q), "l"(a.c.mass + at) : "memory");
            pos[k] = a.recent > 0 ? load<L2>(reinterpret_cast<const int4*>(a.c.positions + at)) : make_int4(0, 0, 0, 0);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");     // each thread reads only what it copied itself
#pragma unroll
        for (int k = 0; k < kLoadBatch; ++k) {
            const int q = q0 + k * kThreads;
            if (q >= quads) break;
            if (page[k] < 0) s.bad = 1;
            const float4 w = *reinterpret_cast<const float4*>(key + 4 * q);
            const float wk[4] = {w.x, w.y, w.z, w.w};
            const int pk[4] = {pos[k].x, pos[k].y, pos[k].z, pos[k].w};
            uint32_t x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = a.recent > 0 && pk[j] >= recent_from ? kKeyRecent : weight_key(wk[j]);
                if (4 * q + j < count) atomicAdd(&s.hist[0][x[j] >> 21], 1);
            }
            *reinterpret_cast<uint4*>(key + 4 * q) = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }

    // ---- the E-th smallest key
    int left = n - budget;                                   // how many go, among the keys that match `prefix` so far
    uint32_t prefix = 0;
    int shift = 32, in_bin = 0;
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, next = shift - bits;
        int (&hist)[kBins] = s.hist[pass & 1];
        if (pass > 0)                                        // (the first digit was counted as the keys came in)
            for (int q = tid; q < quads; q += kThreads) {
                const uint4 v = *reinterpret_cast<const uint4*>(key + 4 * q);
                const uint32_t k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if ((k[j] >> shift) == prefix && 4 * q + j < count) atomicAdd(&hist[(k[j] >> next) & ((1u << bits) - 1u)], 1);
            }
        __syncthreads();
        {                                                    // sums of 32 bins, so that the cluster reads few of them
            constexpr int kPer = kBins / kThreads, kLanes = 32 / kPer;
            int sum = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum += hist[tid * kPer + i];
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (tid % kLanes == 0) s.coarse[pass & 1][tid / kLanes] = sum;
        }
        sync_ranks();
        if (pass == 0) {                                     // a page that is none: the unit stays as it is
            int bad = 0;
            for (int r = 0; r < ranks; ++r) bad |= cluster.map_shared_rank(&s, r)->bad;
            if (bad != 0) {
                if (rank == 0 && tid == 0) {
                    if (a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
                    a.lengths_out[unit] = n;
                }
                sync_ranks();                                // nobody leaves while its shared memory is read
                return;
            }
        }
        if (warp == 0) {                                     // the group of 32 bins, then the bin: summed over the cluster, prefix by shuffles
            int x = 0, y = 0;
#pragma unroll 4
            for (int r = 0; r < ranks; ++r) {
                const int2 v = reinterpret_cast<const int2*>(cluster.map_shared_rank(&s, r)->coarse[pass & 1])[lane];
                x += v.x; y += v.y;
            }
            int upto = x + y;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += o;
            }
            const int pair = __ffs(__ballot_sync(0xffffffffu, upto >= left)) - 1;         // the last lane's is the number of all that match
            const int before_pair = __shfl_sync(0xffffffffu, upto - x - y, pair), first = __shfl_sync(0xffffffffu, x, pair);
            const bool second = before_pair + first < left;
            const int group = 2 * pair + (second ? 1 : 0), before = before_pair + (second ? first : 0);
            int c = 0;
#pragma unroll 4
            for (int r = 0; r < ranks; ++r) c += cluster.map_shared_rank(&s, r)->hist[pass & 1][group * 32 + lane];
            upto = c;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += o;
            }
            if (before + upto - c < left && left <= before + upto) { s.digit = group * 32 + lane; s.left = left - (before + upto - c); s.in_bin = c; }
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint32_t)s.digit;
        left = s.left; in_bin = s.in_bin;
        shift = next;
        if (left == in_bin) break;                           // all keys of the digit go: the rest of the bits decides nothing
        // the third pass takes the first one's histogram: everybody has read it, or nobody could have passed the second's barrier
        if (pass == 1) {
            for (int i = tid; i < kBins; i += kThreads) s.hist[0][i] = 0;
            __syncthreads();
        }
    }

    // ---- which slots go.  A key whose top bits are below `prefix` goes, one above stays; of those that match, the last `left`.
    const int words = (count + 31) / 32;
    const int per = (words + kThreads - 1) / kThreads;       // a run of words per thread, so that its prefix is its run's
    const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
    const int stay = in_bin - left;                          // matching slots that stay: the lowest ones
    const uint32_t rest = shift == 0 ? 0u : (1u << shift) - 1u;
    const uint32_t first_match = prefix << shift, last_match = first_match | rest;
    if (stay == 0) {                                         // everything up to last_match goes
#pragma unroll 4
        for (int w = warp; w < words; w += kWarps) {
            const uint32_t k = key[w * 32 + lane];           // (behind `count` up to a quad's end: masked below)
            const uint32_t m = __ballot_sync(0xffffffffu, k <= last_match);
            if (lane == 0) s.evicted[w] = m;
        }
        __syncthreads();
    } else {                                                 // equal keys on both sides of the line: rank them by slot
        for (int w = warp; w < words; w += kWarps) {
            const uint32_t k = key[w * 32 + lane];
            const bool in = w * 32 + lane < count;
            const uint32_t less = __ballot_sync(0xffffffffu, in && k < first_match);
            const uint32_t same = __ballot_sync(0xffffffffu, in && k >= first_match && k <= last_match);
            if (lane == 0) { s.evicted[w] = less; s.same[w] = same; }
        }
        __syncthreads();
        int at = 0, dummy = 0, tot, tot2;
        for (int w = w0; w < w1; ++w) at += __popc(s.same[w]);
        block_prefix2<kThreads>(s, at, dummy, tot, tot2);
        if (tid == 0) s.ties = tot;
        sync_ranks();
        for (int r = 0; r < rank; ++r) at += cluster.map_shared_rank(&s, r)->ties;
        for (int w = w0; w < w1; ++w) {
            uint32_t m = s.same[w];
            for (; m != 0u && at < stay; ++at) m &= m - 1u;  // these stay
            at += __popc(m);
            s.evicted[w] |= m;
        }
    }

    // ---- lists, in the place of the keys: this slice's holes, then its movers
    auto split = [&](int w, uint32_t& hole, uint32_t& mover) {
        const int first = lo + w * 32;                       // slots [first, first + 32) against the budget
        const uint32_t front = budget >= first + 32 ? 0xffffffffu : budget <= first ? 0u : (1u << (budget - first)) - 1u;
        const uint32_t live = count - w * 32 >= 32 ? 0xffffffffu : (1u << (count - w * 32)) - 1u;
        hole = s.evicted[w] & front & live;
        mover = ~s.evicted[w] & ~front & live;
    };
    int holes = 0, movers = 0, n_holes, n_movers;
    for (int w = w0; w < w1; ++w) {
        uint32_t h, m;
        split(w, h, m);
        holes += __popc(h); movers += __popc(m);
    }
    block_prefix2<kThreads>(s, holes, movers, n_holes, n_movers);      // (its barriers also end the reading of the keys)
    for (int w = w0; w < w1; ++w) {
        uint32_t h, m;
        split(w, h, m);
        for (; h != 0u; h &= h - 1u) key[holes++] = lo + w * 32 + __ffs(h) - 1;
        for (; m != 0u; m &= m - 1u) key[n_holes + movers++] = lo + w * 32 + __ffs(m) - 1;
    }
    if (tid == 0) { s.holes = n_holes; s.movers = n_movers; }
    sync_ranks();
    if (tid < ranks) {
        const EvictShared<kThreads>* o = cluster.map_shared_rank(&s, tid);
        s.rank_holes[tid] = o->holes; s.rank_movers[tid] = o->movers;
    }
    __syncthreads();

    // ---- rows: the cluster's CTAs share the unit's moves.  Batch by batch the threads look up one move each (and move its weight
    // and position), then the warps copy the rows.
    int total = 0;
    for (int r = 0; r < ranks; ++r) total += s.rank_holes[r];
    const int j0 = (int)((long long)rank * total / ranks), j1 = (int)((long long)(rank + 1) * total / ranks);
    const int piece = lane & 15;
    __nv_bfloat16* pool = lane < 16 ? a.c.k : a.c.v;
    for (int jb = j0; jb < j1; jb += kThreads) {
        const int batch = min(kThreads, j1 - jb);
        if (tid < batch) {
            int jh = jb + tid, jm = jh, rh = 0, rm = 0;
            while (jh >= s.rank_holes[rh]) jh -= s.rank_holes[rh++];
            while (jm >= s.rank_movers[rm]) jm -= s.rank_movers[rm++];
            const int to = (int)cluster.map_shared_rank(key, rh)[jh];
            const int from = (int)cluster.map_shared_rank(key, rm)[s.rank_holes[rm] + jm];
            const int from_page = page_of<L2>(a.c, unit, from), to_page = page_of<L2>(a.c, unit, to);
            move[tid] = make_int4(from_page, from, to_page, to);
            const long long f = slot_in_pool(a.c, from_page, from), t = slot_in_pool(a.c, to_page, to);
            const float w = load<L2>(a.c.mass + f);
            const int pos = a.c.positions != nullptr ? load<L2>(a.c.positions + f) : 0;
            a.c.mass[t] = w;
            if (a.c.positions != nullptr) a.c.positions[t] = pos;
        }
        __syncthreads();
        for (int i = warp * kRowBatch; i < batch; i += kWarps * kRowBatch) {
            uint4 x[kRowBatch];
            long long to[kRowBatch];
#pragma unroll
            for (int k = 0; k < kRowBatch; ++k) {
                const int4 mv = move[min(i + k, batch - 1)];       // loads without a condition stay in flight together
                x[k] = load<L2>(reinterpret_cast<const uint4*>(pool + row_in_pool(a.c, mv.x, mv.y)) + piece);
                to[k] = row_in_pool(a.c, mv.z, mv.w);
            }
#pragma unroll
            for (int k = 0; k < kRowBatch; ++k) {
                if (i + k >= batch) break;
                *(reinterpret_cast<uint4*>(pool + to[k]) + piece) = x[k];
            }
        }
        __syncthreads();
    }
    if (rank == 0 && tid == 0) a.lengths_out[unit] = budget;
    sync_ranks();                                            // the lists are read across the cluster until here
}

// kEvictShort runs beside a launch for the long units, which holds it back only from ending: what came before that launch is
// complete when it lets this one start (which reads from L2, where all of that is), and the two touch different units.  (A length
// that the other launch has already replaced, where lengths_out is lengths, reads as a unit at its budget, which stays as it is.)
template <int kThreads, int PART>
__global__ void __launch_bounds__(kThreads, kThreads == kSmallThreads ? 4 : 1)
evict_kernel(const __grid_constant__ EvictArgs a, int slice_cap) {
    if (PART != kEvictShort) pdl_wait();
    pdl_trigger();
    evict_unit<kThreads, PART == kEvictShort>(a, slice_cap, PART);
    if (PART == kEvictShort) pdl_wait();
}

// How many clusters of `ranks` CTAs of the kernel run at once on the current device.  Asked once per kernel, size and device: CTAs of the
// large kernel take an SM each, whatever their slice.
template <int kThreads, int PART>
int clusters_that_fit(cudaLaunchConfig_t cfg, int ranks) {
    const auto kernel = evict_kernel<kThreads, PART>;
    static std::atomic<int> known[64][kMaxCluster + 1];      // 1 more than the number; 0: not asked yet
    int dev = 0, fit = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= 64) return 0;
    if (const int k = known[dev][ranks].load(std::memory_order_relaxed)) return k - 1;
    cfg.gridDim = dim3((unsigned)ranks);
    cfg.dynamicSmemBytes = kLargeSlice * sizeof(uint32_t);
    if ((ranks > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
        cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        fit = 0;
    }
    known[dev][ranks].store(fit + 1, std::memory_order_relaxed);
    return fit;
}

template <int kThreads, int PART>
cudaError_t launch_evict(const EvictArgs& a, int ranks, int least, int max_length, cudaStream_t stream) {
    const auto kernel = evict_kernel<kThreads, PART>;
    static std::atomic<unsigned long long> done;
    cudaError_t e = allow_smem(kernel, (kThreads == kSmallThreads ? kSmallSlice : kLargeSlice) * (int)sizeof(uint32_t), done);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.blockDim = dim3(kThreads); cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled(kPdlOther) ? 2 : 1;
    int slice_cap = 0;
    for (;; ranks = max(least, ranks - 2)) {
        slice_cap = ((max_length + ranks - 1) / ranks + 31) / 32 * 32;
        cfg.gridDim = dim3((unsigned)(a.units * ranks));
        cfg.dynamicSmemBytes = sizeof(uint32_t) * (size_t)slice_cap;
        attr[0].val.clusterDim.x = ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        if (ranks <= least) break;
        // larger clusters than the slices ask for pay only if all units get theirs at once, which the GPU's parts of 16 to 20 SMs may
        // not allow (16 units of 40400 tokens: 27.7 us with clusters of 8, of which not all fit, 18.5 with the largest that do)
        if (clusters_that_fit<kThreads, PART>(cfg, ranks) >= a.units) break;
    }
    e = cudaLaunchKernelEx(&cfg, kernel, a, slice_cap);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_fill(const FillArgs& a, const FillTables& t, cudaStream_t stream) {
    const bool across = a.head_offsets != nullptr;
    const long long rows = (long long)(t.cu_keep[a.nb] - t.cu_keep[0]) * (across ? a.c.heads : 1);
    const bool lengths = a.lengths_out != nullptr || a.status != nullptr, apart = lengths && (rows == 0 || a.lengths_out == a.lengths);
    if (rows > 0) {
        const int row_blocks = (int)((rows + kFillRows - 1) / kFillRows);
        const dim3 grid((unsigned)(row_blocks + (lengths && !apart ? 1 : 0)), across ? a.layers : a.layers * a.c.heads);
        const cudaError_t e = launch_chained(kPdlOther, across ? fill_kernel<true> : fill_kernel<false>, grid, dim3(kFillThreads), 0, stream,
                                             a, t, row_blocks);
        if (e != cudaSuccess) return e;
    }
    if (!apart) return cudaSuccess;
    const long long units = (long long)a.layers * a.c.heads * a.nb;
    return launch_chained(kPdlOther, fill_lengths_kernel, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, stream, a, t);
}

int evict_max_tokens() { return 8 * kLargeSlice; }

cudaError_t launch_paged_evict(const EvictArgs& a, int sm_count, cudaStream_t stream) {
    // Many units: CTAs of 256 threads, four to an SM; where some units may need several CTAs, those go in a launch of clusters, the others
    // in one of single CTAs beside it (one launch of clusters for all left most of their CTAs without work: 128 of 512 ragged
    // units of up to 32768 tokens 56 us against 49).  Few units or very long ones: CTAs of 512 threads, more of them per unit while
    // the GPU is not full and a slice still has 4096 slots (with 2048: 8 units of 5000 tokens 14.1 us against 12.1, 2 of 49169 17.8 against
    // 15.9; with 8192: 8 units of 20000 16.0 us against 14.0, 32 of 20000 17.4 against 16.0, though 32 of 12000 15 against 16).  `least` is
    // where the search for a cluster that fits ends: slices of at most 12288 slots up to clusters of eight (of 6144: 16 units of 30000 tokens
    // 25.6 us against 16.3, since clusters of eight do not all fit; of 24576: no difference in any case tried).
    const int n = a.max_length;
    cudaError_t e;
    if (n <= 8 * kSmallSlice && (long long)a.units * 8 > 2 * sm_count) {
        if (n <= kSmallSlice) return launch_evict<kSmallThreads, kEvictAll>(a, 1, 1, n, stream);
        int ranks = 2;
        while (n > ranks * kSmallSlice) ranks *= 2;
        e = launch_evict<kSmallThreads, kEvictLong>(a, ranks, ranks, n, stream);
        return e != cudaSuccess ? e : launch_evict<kSmallThreads, kEvictShort>(a, 1, 1, kSmallSlice, stream);
    }
    int least = 1;
    while (least < 8 && n > (long long)least * 12288) least *= 2;
    int ranks = least;
    while (ranks < kMaxCluster && (long long)a.units * ranks * 2 <= sm_count && n > 8192LL * ranks) ranks *= 2;
    return launch_evict<kLargeThreads, kEvictAll>(a, ranks, least, n, stream);
}

}  // namespace compactor
