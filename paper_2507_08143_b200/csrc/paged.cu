// The paged cache's two copying operators: filling pages with the rows that a selection kept, and evicting the tokens of
// least accumulated attention weight.  Both move whole 256-byte rows as 16-byte pieces, bit for bit.
#include "paged.cuh"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace compactor {
namespace {

// ------------------------------------------------------------------------------------------ fill
// 16 threads per row as in the dense gather (compact.cu); what is new is where a row goes: slot lengths[unit] + j of
// its unit, j its place among the unit's kept rows, found through the page table.  Bound by HBM: 512 bytes read and
// written per row.
constexpr int kFillThreads = 256;
constexpr int kFillRowsPerIter = kFillThreads / 16;
constexpr int kFillSteps = 8;
constexpr int kFillRows = kFillRowsPerIter * kFillSteps;

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n"
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
    const int n = a.lengths != nullptr ? __ldg(a.lengths + unit) : 0;
    if (n < 0) return -1;
    return (long long)n + rows > ((long long)a.c.max_pages << a.c.page_shift) ? -1 : n;
}

template <bool ACROSS>
__global__ void __launch_bounds__(kFillThreads)
fill_kernel(const __grid_constant__ FillArgs a, const __grid_constant__ FillTables t) {
    const int piece = threadIdx.x & 15, sub = threadIdx.x >> 4;
    const int layer = ACROSS ? blockIdx.y : blockIdx.y / a.c.heads;
    const long long per_outer = ACROSS ? (long long)a.c.heads * a.total_keep : a.total_keep;     // rows per layer or (layer, head)
    const long long scale = ACROSS ? a.c.heads : 1;
    const long long end = scale * t.cu_keep[a.nb];
    const long long row0 = scale * t.cu_keep[0] + (long long)blockIdx.x * kFillRows;
#pragma unroll
    for (int step = 0; step < kFillSteps; ++step) {
        const long long row = row0 + step * kFillRowsPerIter + sub;
        if (row >= end) return;
        const int b = find_segment(t.cu_keep, a.nb, (int)(row / scale));
        int head, j;
        if (ACROSS) {
            const int* offs = a.head_offsets + ((long long)layer * a.c.batch + a.b0 + b) * (a.c.heads + 1);
            j = (int)(row - scale * t.cu_keep[b]);
            head = find_segment(offs, a.c.heads, j);
            j -= offs[head];
        } else {
            head = blockIdx.y - layer * a.c.heads;
            j = (int)row - t.cu_keep[b];
        }
        const int n = t.cu_seqlens[b + 1] - t.cu_seqlens[b];
        const int local = a.idx != nullptr ? __ldg(a.idx + (long long)blockIdx.y * per_outer + row) : j;
        const int unit = ((a.first_layer + layer) * a.c.heads + head) * a.c.batch + a.b0 + b;
        const int rows = kept_rows(a, t, layer, head, b), first = first_slot(a, unit, rows);
        if (first < 0 || j < 0 || j >= rows || (unsigned)local >= (unsigned)n) continue;
        const int slot = first + j;
        const int page = page_of(a.c, unit, slot);
        if (page < 0) {
            if (piece == 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
            continue;
        }
        const long long tok = (long long)t.cu_seqlens[b] + local;
        const long long to = row_in_pool(a.c, page, slot);
        const uint4 kv = ld_stream(reinterpret_cast<const uint4*>(a.k.ptr + layer * a.k.stride_layer + head * a.k.stride_head +
                                                                  tok * a.k.stride_token) + piece);
        const uint4 vv = ld_stream(reinterpret_cast<const uint4*>(a.v.ptr + layer * a.v.stride_layer + head * a.v.stride_head +
                                                                  tok * a.v.stride_token) + piece);
        reinterpret_cast<uint4*>(a.c.k + to)[piece] = kv;
        reinterpret_cast<uint4*>(a.c.v + to)[piece] = vv;
        if (piece == 0 && a.c.mass != nullptr)
            a.c.mass[slot_in_pool(a.c, page, slot)] =
                a.mass_in != nullptr ? a.mass_in[((long long)layer * a.c.heads + head) * a.total_tokens + tok] : 0.f;
        if (piece == 1 && a.c.positions != nullptr)
            a.c.positions[slot_in_pool(a.c, page, slot)] = (a.first_position != nullptr ? a.first_position[a.b0 + b] : 0) + local;
    }
}

// New lengths, and the units that had no room.  A launch of its own: lengths_out may be lengths, which every block of the
// fill reads.
__global__ void fill_lengths_kernel(const __grid_constant__ FillArgs a, const __grid_constant__ FillTables t) {
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (long long)a.layers * a.c.heads * a.nb) return;
    const int b = (int)(i % a.nb), lh = (int)(i / a.nb), layer = lh / a.c.heads, head = lh - layer * a.c.heads;
    const int unit = ((a.first_layer + layer) * a.c.heads + head) * a.c.batch + a.b0 + b;
    const int rows = kept_rows(a, t, layer, head, b), first = first_slot(a, unit, rows);
    const int n = a.lengths != nullptr ? a.lengths[unit] : 0;
    if (first < 0 && n >= 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
    if (a.lengths_out != nullptr) a.lengths_out[unit] = first < 0 ? n : n + rows;
}

// ------------------------------------------------------------------------------------------ evict
// One cluster of 1 to 8 CTAs per unit; each CTA holds the sort keys of a slice of the unit's slots in shared memory.
//   key      the weight as an ordered 32-bit integer; the largest key for a recent token (never below a weight)
//   1. radix selection of the E-th smallest key, E = n - budget: digits of 11, 11 and 10 bits, one histogram per CTA,
//      summed over the cluster through distributed shared memory by every CTA alike
//   2. a bit per slot: evicted or not (of equal keys the higher slots go first)
//   3. lists of the holes (evicted, below the budget) and the movers (kept, at or above it), both ascending; there are as
//      many of one as of the other, and the j-th mover's row goes to the j-th hole.  Sources and targets never overlap, so the
//      rows move in any order, and no more than min(E, budget) of them move: compaction that kept the slots' order
//      would rewrite nearly the whole unit for one evicted token.
// Bound by HBM (8 bytes per slot, 1 KB per moved row) for many units; for few or small ones by the chain of block-wide steps.
constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 49152;                // slots per CTA: 192 KB of keys
constexpr int kMaxWords = kMaxSlice / 32;
constexpr uint32_t kKeyRecent = 0xffffffffu, kKeyNan = 0xfffffffeu;

struct EvictShared {
    int hist[kBins];
    uint32_t evicted[kMaxWords];                // bit per slot of the slice
    uint32_t same[kMaxWords];                   // bit per slot whose key cannot be told from the E-th smallest
    int warp_a[kEvictWarps], warp_b[kEvictWarps];
    int holes, movers, ties, bad;               // of this CTA's slice
    int digit, left, in_bin;
};

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return kKeyNan;                 // as in the selection of the prefill: not a number ranks above +inf
    const uint32_t u = __float_as_uint(w + 0.f);             // -0 is 0
    return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}

// Exclusive prefix over the block of two counts per thread, and their totals.
__device__ __forceinline__ void block_prefix2(EvictShared& s, int& x, int& y, int& total_x, int& total_y) {
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
    for (int w = 0; w < kEvictWarps; ++w) {
        const int cx = s.warp_a[w], cy = s.warp_b[w];
        if (w < warp) { bx += cx; by += cy; }
        total_x += cx; total_y += cy;
    }
    x = bx + ix - x; y = by + iy - y;
}

__global__ void __launch_bounds__(kEvictThreads, 1)
evict_kernel(const __grid_constant__ EvictArgs a, int slice_cap) {
    extern __shared__ __align__(16) uint32_t key[];          // [slice_cap]; afterwards the two lists
    __shared__ __align__(16) EvictShared s;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int unit = a.first_unit + (int)(blockIdx.x / ranks);
    const int n = a.lengths[unit], budget = a.budgets[unit];
    const long long capacity = min((long long)a.max_length, (long long)a.c.max_pages << a.c.page_shift);
    // nothing to do: the same decision in every CTA of the cluster, before any barrier between them
    if (n < 0 || budget < 0 || n <= budget || n > capacity || budget == 0) {
        if (rank == 0 && tid == 0) {
            const bool refused = n > capacity;
            if (refused && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
            a.lengths_out[unit] = !refused && budget == 0 && n > 0 ? 0 : n;
        }
        return;
    }
    const int slice = ((n + ranks - 1) / ranks + 31) / 32 * 32;              // at most slice_cap: n <= max_length
    const int lo = min(n, rank * slice), count = min(n, lo + slice) - lo;
    const int recent_from = a.recent > 0 ? a.next_position[unit % a.c.batch] - min(a.recent, budget) : 0;

    if (tid == 0) s.bad = 0;
    __syncthreads();
    for (int i = tid; i < count; i += kEvictThreads) {
        const int page = page_of(a.c, unit, lo + i);
        uint32_t k = 0;
        if (page < 0) s.bad = 1;
        else {
            const long long at = slot_in_pool(a.c, page, lo + i);
            k = weight_key(a.c.mass[at]);
            if (a.recent > 0 && a.c.positions[at] >= recent_from) k = kKeyRecent;
        }
        key[i] = k;
    }

    // ---- the E-th smallest key
    int left = n - budget;                                   // how many go, among the keys that match `prefix` so far
    uint32_t prefix = 0;
    int shift = 32, in_bin = 0;
    bool whole_bin = false;
    for (int pass = 0; pass < 3 && !whole_bin; ++pass) {
        const int bits = pass < 2 ? 11 : 10, next = shift - bits;
        for (int i = tid; i < kBins; i += kEvictThreads) s.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < count; i += kEvictThreads) {
            const uint32_t k = key[i];
            if (pass == 0 || (k >> shift) == prefix) atomicAdd(&s.hist[(k >> next) & ((1u << bits) - 1u)], 1);
        }
        cluster.sync();
        if (pass == 0) {                                     // a page that is none: the unit stays as it is
            int bad = 0;
            for (int r = 0; r < ranks; ++r) bad |= cluster.map_shared_rank(&s, r)->bad;
            if (bad != 0) {
                if (rank == 0 && tid == 0) {
                    if (a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
                    a.lengths_out[unit] = n;
                }
                cluster.sync();                              // nobody leaves while its shared memory is read
                return;
            }
        }
        constexpr int kPer = kBins / kEvictThreads;
        int c[kPer], sum = 0, dummy = 0, tot, tot2;
#pragma unroll
        for (int i = 0; i < kPer; ++i) c[i] = 0;
        for (int r = 0; r < ranks; ++r) {
            const int4 v = *reinterpret_cast<const int4*>(&cluster.map_shared_rank(&s, r)->hist[tid * kPer]);
            c[0] += v.x; c[1] += v.y; c[2] += v.z; c[3] += v.w;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += c[i];
        int before = sum;
        block_prefix2(s, before, dummy, tot, tot2);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (before < left && left <= before + c[i]) { s.digit = tid * kPer + i; s.left = left - before; s.in_bin = c[i]; }
            before += c[i];
        }
        cluster.sync();                                      // the histograms have been read everywhere; s.digit is there
        prefix = (prefix << bits) | (uint32_t)s.digit;
        left = s.left; in_bin = s.in_bin;
        shift = next;
        whole_bin = left == in_bin;                          // the rest of the digits decides nothing
        __syncthreads();
    }

    // ---- which slots go.  A key whose top bits are below `prefix` goes, one above stays; of those that match, the last `left`.
    const int words = (count + 31) / 32;
    const int per = (words + kEvictThreads - 1) / kEvictThreads;             // a run of words per thread, so that its prefix is its run's
    const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
    const int stay = in_bin - left;                          // matching slots that stay: the lowest ones
    for (int w = warp; w < words; w += kEvictWarps) {
        const int i = w * 32 + lane;
        const uint32_t top = i < count ? (shift == 0 ? key[i] : key[i] >> shift) : 0xffffffffu;
        const uint32_t less = __ballot_sync(0xffffffffu, i < count && top < prefix);
        const uint32_t same = __ballot_sync(0xffffffffu, i < count && top == prefix);
        if (lane == 0) { s.evicted[w] = stay == 0 ? less | same : less; s.same[w] = same; }
    }
    __syncthreads();
    if (stay > 0) {                                          // equal keys on both sides of the line: rank them by slot
        int at = 0, dummy = 0, tot, tot2;
        for (int w = w0; w < w1; ++w) at += __popc(s.same[w]);
        block_prefix2(s, at, dummy, tot, tot2);
        if (tid == 0) s.ties = tot;
        cluster.sync();
        for (int r = 0; r < rank; ++r) at += cluster.map_shared_rank(&s, r)->ties;
        for (int w = w0; w < w1; ++w) {
            uint32_t m = s.same[w];
            for (; m != 0u && at < stay; ++at) m &= m - 1u;  // these stay
            at += __popc(m);
            s.evicted[w] |= m;
        }
        __syncthreads();
    }

    // ---- lists, in the place of the keys: this slice's holes, then its movers
    int holes = 0, movers = 0, n_holes, n_movers;
    auto split = [&](int w, uint32_t& hole, uint32_t& mover) {
        const int first = lo + w * 32;                       // slots [first, first + 32) against the budget
        const uint32_t front = budget >= first + 32 ? 0xffffffffu : budget <= first ? 0u : (1u << (budget - first)) - 1u;
        const uint32_t live = count - w * 32 >= 32 ? 0xffffffffu : (1u << (count - w * 32)) - 1u;
        hole = s.evicted[w] & front & live;
        mover = ~s.evicted[w] & ~front & live;
    };
    for (int w = w0; w < w1; ++w) {
        uint32_t h, m;
        split(w, h, m);
        holes += __popc(h); movers += __popc(m);
    }
    block_prefix2(s, holes, movers, n_holes, n_movers);
    for (int w = w0; w < w1; ++w) {
        uint32_t h, m;
        split(w, h, m);
        for (; h != 0u; h &= h - 1u) key[holes++] = lo + w * 32 + __ffs(h) - 1;
        for (; m != 0u; m &= m - 1u) key[n_holes + movers++] = lo + w * 32 + __ffs(m) - 1;
    }
    if (tid == 0) { s.holes = n_holes; s.movers = n_movers; }
    cluster.sync();

    // ---- rows: the cluster's CTAs share the unit's moves
    int total = 0;
    for (int r = 0; r < ranks; ++r) total += cluster.map_shared_rank(&s, r)->holes;
    const int j0 = (int)((long long)rank * total / ranks), j1 = (int)((long long)(rank + 1) * total / ranks);
    auto lookup = [&](int j, bool hole) {
        for (int r = 0; r < ranks; ++r) {
            const EvictShared* o = cluster.map_shared_rank(&s, r);
            const int have = hole ? o->holes : o->movers;
            if (j < have) return (int)cluster.map_shared_rank(key, r)[(hole ? 0 : o->holes) + j];
            j -= have;
        }
        return 0;
    };
    const int piece = lane & 15;
    __nv_bfloat16* pool = lane < 16 ? a.c.k : a.c.v;
    constexpr int kInFlight = 4;
    for (int j = j0 + warp * kInFlight; j < j1; j += kEvictWarps * kInFlight) {
        uint4 x[kInFlight];
        long long to[kInFlight], at[kInFlight];
        float w[kInFlight];
        int pos[kInFlight];
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            const int jj = min(j + i, j1 - 1);               // loads without a condition stay in flight together
            const int from_slot = lookup(jj, false), to_slot = lookup(jj, true);
            const int from_page = page_of(a.c, unit, from_slot), to_page = page_of(a.c, unit, to_slot);
            x[i] = *(reinterpret_cast<const uint4*>(pool + row_in_pool(a.c, from_page, from_slot)) + piece);
            to[i] = row_in_pool(a.c, to_page, to_slot);
            at[i] = slot_in_pool(a.c, to_page, to_slot);
            const long long from = slot_in_pool(a.c, from_page, from_slot);
            w[i] = a.c.mass[from];
            pos[i] = a.c.positions != nullptr ? a.c.positions[from] : 0;
        }
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            if (j + i >= j1) break;
            *(reinterpret_cast<uint4*>(pool + to[i]) + piece) = x[i];
            if (lane == 0) a.c.mass[at[i]] = w[i];
            if (lane == 1 && a.c.positions != nullptr) a.c.positions[at[i]] = pos[i];
        }
    }
    if (rank == 0 && tid == 0) a.lengths_out[unit] = budget;
    cluster.sync();                                          // the lists are read across the cluster until here
}

}  // namespace

cudaError_t launch_paged_fill(const FillArgs& a, const FillTables& t, cudaStream_t stream) {
    const bool across = a.head_offsets != nullptr;
    const long long rows = (long long)(t.cu_keep[a.nb] - t.cu_keep[0]) * (across ? a.c.heads : 1);
    if (rows == 0) return cudaSuccess;
    const dim3 grid((unsigned)((rows + kFillRows - 1) / kFillRows), across ? a.layers : a.layers * a.c.heads);
    if (across) fill_kernel<true><<<grid, kFillThreads, 0, stream>>>(a, t);
    else fill_kernel<false><<<grid, kFillThreads, 0, stream>>>(a, t);
    return cudaGetLastError();
}

cudaError_t launch_paged_fill_lengths(const FillArgs& a, const FillTables& t, cudaStream_t stream) {
    const long long units = (long long)a.layers * a.c.heads * a.nb;
    fill_lengths_kernel<<<(unsigned)((units + 255) / 256), 256, 0, stream>>>(a, t);
    return cudaGetLastError();
}

int evict_max_tokens() { return kMaxCluster * kMaxSlice; }

cudaError_t launch_paged_evict(const EvictArgs& a, int sm_count, cudaStream_t stream) {
    // CTAs per unit: enough for their slices to fit, more while the GPU is not full and a slice still has 2048 slots
    int ranks = 1;
    while (ranks < kMaxCluster && (a.max_length > (long long)ranks * kMaxSlice ||
                                   ((long long)a.units * ranks * 2 <= sm_count && a.max_length > 4096LL * ranks)))
        ranks *= 2;
    const int slice_cap = ((a.max_length + ranks - 1) / ranks + 31) / 32 * 32;
    const size_t smem = sizeof(uint32_t) * (size_t)slice_cap;
    cudaError_t e = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * (int)sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.units * ranks)); cfg.blockDim = dim3(kEvictThreads);
    cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, evict_kernel, a, slice_cap);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace compactor
