// Device-side view of a paged cache (compactor_paged_cache) shared by the kernels that fill, read and evict it.
#pragma once
#include <atomic>

#include "common.cuh"

namespace compactor {

struct Paged {
    __nv_bfloat16* k;
    __nv_bfloat16* v;
    long long stride_page, stride_token;   // elements, the same for K and V
    float* mass;                           // [n_pages][page_tokens] accumulated attention weights, or null
    int* positions;                        // [n_pages][page_tokens], or null
    const int* table;                      // [layers * heads * batch][max_pages]
    int n_pages, max_pages;
    int page_shift;                        // page_tokens = 1 << page_shift
    int layers, heads, batch;
    int row_pieces;                        // 16-byte pieces of a row: 16, or 5 where rows are held in 4 bits (strides are then in units of 2 bytes)
};

// Chained kernels are already running while their predecessor still writes.  What they read after pdl_wait() they read plainly; never
// through the read-only path (ld.global.nc), whose lines may be old.  What a kernel reads before pdl_wait() (because a
// kernel further back in the chain has waited for its writer) it reads from L2 (`L2`).
template <bool L2, typename T> __device__ __forceinline__ T load(const T* p) { return L2 ? __ldcg(p) : *p; }

// Page of slot `slot` of unit `unit`, or -1 where the table holds no page of the pool.  The caller has checked that
// the slot lies within the unit's row of the table.
template <bool L2>
__device__ __forceinline__ int page_of(const Paged& c, int unit, int slot) {
    const int id = load<L2>(c.table + (long long)unit * c.max_pages + (slot >> c.page_shift));
    return (unsigned)id < (unsigned)c.n_pages ? id : -1;
}
// Element offset of a slot's row in the pools, given its page (64 bits: a pool may hold more than 2^32 elements).
__device__ __forceinline__ long long row_in_pool(const Paged& c, int page, int slot) {
    return (long long)page * c.stride_page + (long long)(slot & ((1 << c.page_shift) - 1)) * c.stride_token;
}
// Index of a slot in the weight and position pools.
__device__ __forceinline__ long long slot_in_pool(const Paged& c, int page, int slot) {
    return ((long long)page << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
}

// Dynamic shared memory limit of a kernel, set on its first launch on each device (`done`: a static of the caller; setting it twice
// from two threads does no harm).
template <typename K>
inline cudaError_t allow_smem(K kernel, int bytes, std::atomic<unsigned long long>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (bit != 0 && (done.load(std::memory_order_relaxed) & bit) != 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Sequences per launch of the fill kernel: their prefix tables travel as kernel arguments.
constexpr int kFillSeqs = 256;
struct FillTables { int cu_seqlens[kFillSeqs + 1]; int cu_keep[kFillSeqs + 1]; };
struct FillArgs {
    Paged c;
    Mat k, v;
    int first_layer, layers;               // layers of the cache that the prefill's layers go to
    int b0, nb;                            // sequences of this launch
    int total_tokens, total_keep;          // of the whole call, per (layer, head)
    const int* idx;                        // null: rows 0 .. keep - 1 of every sequence
    const int* head_offsets;               // selection across heads, else null
    const float* mass_in;                  // [layers][heads][total_tokens] or null
    const int* first_position;             // [batch] or null
    const int* lengths;                    // [units of the cache] or null (all empty)
    int* lengths_out;
    int* status;
    int four;                              // rows are held in 4 bits
};
cudaError_t launch_paged_fill(const FillArgs& a, const FillTables& t, cudaStream_t stream);

// One new token per sequence against one layer of the cache.
struct DecodeArgs {
    Paged c;                               // table, lengths and status start at the layer's first unit
    const __nv_bfloat16* q;
    long long q_seq, q_head;
    const __nv_bfloat16* k_new;            // null: nothing is appended
    const __nv_bfloat16* v_new;
    long long kn_seq, kn_head, vn_seq, vn_head;
    const int* new_positions;              // [batch] or null
    const int* lengths;                    // [heads * batch]
    __nv_bfloat16* out;
    long long out_seq, out_head;
    float* lse;                            // [batch][heads * g] or null
    int* status;                           // [heads * batch] or null
    int g;                                 // query heads per KV head
    int groups;                            // ceil(g / 16): a unit's query heads are served 16 at a time
    int capacity;                          // most tokens of a unit, the new one included
    int accumulate;
    float scale, softcap;                  // softcap <= 0: none
    int units;
    int workers;                           // warps that share the tokens
    int busy_workers;                      // the same where each gets many tiles
    int four;                              // rows are held in 4 bits
    int* prefix;                           // workspace: [units + 1] cost before each unit
    float* ml;                             // workspace: [workers + units * groups][2][16] running maximum and sum
    float* o;                              // workspace: [workers + units * groups][min(g, 16)][128]
    float* scores;                         // workspace: [units][g][unit_rows] in base 2, only when accumulating
    int unit_rows;                         // the capacity in whole tiles
};
constexpr int kDecodeTile = 16;            // tokens per tile
constexpr int kDecodeWarps = 8;
constexpr int kDecode4Warps = 12;          // of the kernel for rows in 4 bits, up to 8 query heads (168 registers a thread)
constexpr int kDecode4WarpsWide = 8;       // and beyond
constexpr int kDecodeUnitCost = 3;         // tiles that entering a unit counts for when the work is shared out
constexpr int kDecodeHeads = 16;           // query heads that one warp serves at once
constexpr int kDecodeMassUnitCost = 64;    // the same, in the kernel that adds the weights
cudaError_t launch_paged_attention(const DecodeArgs& a, int sm_count, cudaStream_t stream);
cudaError_t launch_decode4(const DecodeArgs& a, cudaStream_t stream);     // its first kernel for rows in 4 bits

// Rows out of the pages into dense tensors.
struct ReadTables { int cu_seqlens[kFillSeqs + 1]; };
struct ReadArgs {
    Paged c;
    __nv_bfloat16* k;
    __nv_bfloat16* v;
    long long k_layer, k_head, k_token, v_layer, v_head, v_token;
    int first_layer, layers;
    int b0, nb;                            // sequences of this launch
    const int* first;                      // [units of the cache] or null (0)
    const int* lengths;
    int* status;
    int four;
};
cudaError_t launch_paged_read(const ReadArgs& a, const ReadTables& t, cudaStream_t stream);

// Least and greatest key of every page.
struct BoundsArgs {
    Paged c;
    int first_unit, units;
    int capacity;                          // most tokens of a unit
    const int* first;                      // [units of the cache] or null (0): pages before this token's stay as they are
    const int* lengths;
    __nv_bfloat16* bounds;                 // [n_pages][2][128]
    int* status;
    int four;
};
cudaError_t launch_paged_bounds(const BoundsArgs& a, int sm_count, cudaStream_t stream);

// Choice of pages for the queries of one new token per sequence.
struct SelectArgs {
    Paged c;                               // table, lengths and status start at the layer's first unit
    const __nv_bfloat16* q;
    long long q_seq, q_head;
    const __nv_bfloat16* k_new;            // null: nothing is going to be appended
    long long kn_seq, kn_head;
    const int* lengths;
    __nv_bfloat16* bounds;
    int* table_out;                        // [units][pages]
    int* lengths_out;                      // [units]
    int* status;
    uint32_t* keys;                        // workspace: [units][unit_pages] scores, as ordered integers
    float* errors;                         // workspace: [units][unit_pages] how far they may be off
    int g, units, capacity, unit_pages;
    int pages, first_pages, last_pages;
};
constexpr int kSelectMaxPages = 49152;     // most pages of a unit: their keys lie in shared memory
cudaError_t launch_paged_select(const SelectArgs& a, int sm_count, cudaStream_t stream);

struct EvictArgs {
    Paged c;
    int first_unit, units;
    const int* lengths;
    const int* budgets;
    const int* next_position;              // [batch], null when recent = 0
    int recent;
    int max_length;
    int* lengths_out;
    int* status;
};
int evict_max_tokens();                    // longest unit the kernel takes
cudaError_t launch_paged_evict(const EvictArgs& a, int sm_count, cudaStream_t stream);

}  // namespace compactor
