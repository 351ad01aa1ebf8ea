// Rows out of the pages of a cache into dense tensors, the counterpart of the fill: token first[u] + j of a unit goes to row cu_seqlens[b] + j of
// its (layer, head).  Rows held in 4 bits come out as the bf16 nearest to lo + s c.
//
// Bound by HBM: 512 or 160 bytes read and 512 written per token.  A block moves 128 rows: a thread per row finds its source (length and
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
// Least and greatest key of a page, channel by channel, over its tokens: what the choice of pages goes by.  Bound by HBM: 256 (80) bytes per
// token.  16 lanes hold a row; a warp has 16 rows in flight (32 in 4 bits, which are fewer bytes), and the least and greatest of a lane's eight
// channels stay packed (min and max of bf16 are exact; they keep a not-a-number).  A warp takes a whole page where there are enough pages for all
// warps of the GPU, so that its chain of reads (length, page id, rows) is made once; up to eight share one where there are few.
constexpr int kBoundsThreads = 256;

template <bool FOUR>
__global__ void __launch_bounds__(kBoundsThreads)
bounds_kernel(const __grid_constant__ BoundsArgs a, int chunks, int warps_per_page) {
    __shared__ uint4 part[kBoundsThreads / 32][2][16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, piece = lane & 15;
    pdl_trigger();
    pdl_wait();
    const int unit = a.first_unit + blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const int n = a.lengths[unit];
    if (n < 0) return;
    if (n > a.capacity) {
        if (tid == 0 && chunk == 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_CAPACITY);
        return;
    }
    const int first = a.first != nullptr ? max(0, a.first[unit]) : 0;
    const int index = chunk * (kBoundsThreads / 32 / warps_per_page) + warp / warps_per_page;        // of the unit's pages
    const long long slot0 = (long long)index << a.c.page_shift;
    const bool mine = slot0 < n && index >= first >> a.c.page_shift;
    int page = -1;
    if (mine) {
        page = page_of<false>(a.c, unit, (int)slot0);
        if (page < 0 && lane == 0 && a.status != nullptr) atomicOr(a.status + unit, COMPACTOR_STATUS_PAGE);
    }
    uint32_t least[4], most[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { least[i] = 0x7f807f80u; most[i] = 0xff80ff80u; }
    if (page >= 0) {
        const int tokens = (int)min((long long)1 << a.c.page_shift, n - slot0);
        constexpr int kBatch = FOUR ? 16 : 8;                // pairs of rows in flight
        const int way = warp % warps_per_page;               // every warps_per_page-th run of rows, from the way-th on
        const long long row0 = row_in_pool(a.c, page, 0);
#pragma unroll 1
        for (int r0 = 2 * kBatch * way; r0 < tokens; r0 += 2 * kBatch * warps_per_page) {
            uint4 x[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {               // (a row behind the last: the last once more)
                const __nv_bfloat16* row = a.c.k + row0 + min(r0 + 2 * i + (lane >> 4), tokens - 1) * a.c.stride_token;
                if (FOUR) {
                    const unsigned char* src = reinterpret_cast<const unsigned char*>(row);
                    x[i].x = *reinterpret_cast<const uint32_t*>(src + 4 * piece);
                    x[i].y = *reinterpret_cast<const uint32_t*>(src + kRow4Codes + (piece & ~3));
                } else {
                    x[i] = *(reinterpret_cast<const uint4*>(row) + piece);
                }
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                if (FOUR) {                                  // pairs of channels four apart
                    const uint32_t s = __byte_perm(x[i].y, 0u, 0x1010), lo = __byte_perm(x[i].y, 0u, 0x3232);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = fma2(fma2(codes128(x[i].x, j), 0x3f803f80u, 0xc300c300u), s, lo);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) { least[j] = min_nan2(least[j], w[j]); most[j] = max_nan2(most[j], w[j]); }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        least[j] = min_nan2(least[j], __shfl_xor_sync(0xffffffffu, least[j], 16));
        most[j] = max_nan2(most[j], __shfl_xor_sync(0xffffffffu, most[j], 16));
    }
    if (warps_per_page > 1) {
        if (lane < 16) {
            part[warp][0][piece] = make_uint4(least[0], least[1], least[2], least[3]);
            part[warp][1][piece] = make_uint4(most[0], most[1], most[2], most[3]);
        }
        __syncthreads();
        if (warp % warps_per_page != 0) return;
        for (int o = 1; o < warps_per_page; ++o) {
            const uint4 l = part[warp + o][0][piece], m = part[warp + o][1][piece];
            least[0] = min_nan2(least[0], l.x); least[1] = min_nan2(least[1], l.y); least[2] = min_nan2(least[2], l.z); least[3] = min_nan2(least[3], l.w);
            most[0] = max_nan2(most[0], m.x); most[1] = max_nan2(most[1], m.y); most[2] = max_nan2(most[2], m.z); most[3] = max_nan2(most[3], m.w);
        }
    }
    if (page < 0) return;
    uint4 out = lane < 16 ? make_uint4(least[0], least[1], least[2], least[3]) : make_uint4(most[0], most[1], most[2], most[3]);
    if (FOUR)                                                // channels back in their order
        out = make_uint4(__byte_perm(out.x, out.y, 0x5410), __byte_perm(out.z, out.w, 0x5410), __byte_perm(out.x, out.y, 0x7632), __byte_perm(out.z, out.w, 0x7632));
    *(reinterpret_cast<uint4*>(a.bounds + (long long)page * 2 * kD + (lane >> 4) * kD) + piece) = out;
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
    int warps_per_page = 1;
    while (warps_per_page < 8 && page > (a.four ? 32 : 16) * warps_per_page && (long long)a.units * pages * warps_per_page < 64LL * sm_count) warps_per_page *= 2;
    const int per_block = 8 / warps_per_page, chunks = (pages + per_block - 1) / per_block;
    return launch_chained(kPdlOther, a.four ? bounds_kernel<true> : bounds_kernel<false>, dim3((unsigned)(a.units * chunks)), dim3(kBoundsThreads), 0,
                          stream, a, chunks, warps_per_page);
}

}  // namespace compactor
