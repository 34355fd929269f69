// What the calls on a paged cache share: their arguments as the kernels take them, and how a table is read.
#pragma once

#include "common.cuh"

namespace sc {
namespace pg {

// A cache as the kernels take it (T the storage type; strides in elements).
template <typename T>
struct Pages {
    T* k; T* v; int32_t* count; T* k_min; T* k_max;
    const int32_t* table;
    int64_t page_stride, head_stride, row_stride, table_stride;
    int num_pages, page_size, page_heads, table_heads, max_pages;

    __host__ __device__ int cap() const { return max_pages * page_size; }
    __device__ const int32_t* table_of(int entry) const { return table + entry * table_stride; }   // entry = b * table_heads + ht
    __device__ bool names_page(int id) const { return (unsigned)id < (unsigned)num_pages; }
};

template <typename T>
inline Pages<T> pages_of(const sc_paged_cache& c) {
    Pages<T> p;
    p.k = (T*)c.k; p.v = (T*)c.v; p.count = c.count; p.k_min = (T*)c.k_min; p.k_max = (T*)c.k_max;
    p.table = c.table; p.page_stride = c.page_stride; p.head_stride = c.head_stride; p.row_stride = c.row_stride;
    p.table_stride = c.table_stride; p.num_pages = c.num_pages; p.page_size = c.page_size; p.page_heads = c.page_heads;
    p.table_heads = c.table_heads; p.max_pages = c.max_pages;
    return p;
}

// ---- how attention's work is shared out ----------------------------------------------------
// The rows of every head, in tiles, form one line: entry after entry of `lens`, its heads (and groups of query heads: "units")
// after one another.  A launch's parties (blocks, or clusters of blocks) take equal stretches of it, so that a batch is
// balanced whatever its lengths are, and nothing about them has to be known on the host.  A party's stretch is cut into
// segments at the units' ends.  A unit inside one stretch is finished there; the parties that share one leave partial sums,
// each in one of two slots of its own (the unit its stretch begins in, and the one it ends in), and the last to arrive joins them.
// Arrival counters, one per party (the first of those that share a unit), lie at the front of the workspace in a place of the same size
// for every shape and kernel, so that no call's partial sums lie where another one's counters are.
constexpr size_t kTicketBytes = 4096;
struct Line {
    const int32_t* lens;
    int entries, per_entry, cap, tile, parties;   // per_entry: units of an entry

    __device__ __forceinline__ int len(int e) const { return max(min(lens[e], cap), 0); }
    __device__ __forceinline__ int tiles(int e) const { return (len(e) + tile - 1) / tile; }
};
struct Place {              // a position on the line
    int entry, unit, tile;
    int64_t at;             // of the unit's first tile
};

// Length of a party's stretch.  All lanes of a warp call it; every warp of the launch gets the same.
__device__ __forceinline__ int64_t stretch_of(const Line& line, int least, int lane, int64_t& total) {
    int64_t sum = 0;
#pragma unroll 4
    for (int e = lane; e < line.entries; e += 32) sum += line.tiles(e);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
    total = sum * line.per_entry;
    const int64_t each = (total + line.parties - 1) / line.parties;
    return each > least ? each : least;
}

// The place of tile `at` of the line (at < total).  All lanes of a warp call it.
__device__ __forceinline__ Place place_of(const Line& line, int64_t at, int lane) {
    int64_t before = 0;
    for (int e0 = 0;; e0 += 32) {
        const int nt = e0 + lane < line.entries ? line.tiles(e0 + lane) : 0;
        const int64_t mine = (int64_t)nt * line.per_entry;
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += t;
        }
        const unsigned past = __ballot_sync(kFull, before + upto > at);
        if (past != 0) {
            const int src = __ffs(past) - 1;
            const int64_t start = before + __shfl_sync(kFull, upto - mine, src);
            const int t = __shfl_sync(kFull, nt, src);
            Place p;
            p.entry = e0 + src;
            p.unit = (int)((at - start) / t);
            p.at = start + (int64_t)p.unit * t;
            p.tile = (int)(at - p.at);
            return p;
        }
        before += __shfl_sync(kFull, upto, 31);
    }
}

// The next unit that has tiles (one follows: the caller has tiles left).
__device__ __forceinline__ void next_unit(const Line& line, Place& p, int tiles_here) {
    p.at += tiles_here;
    p.tile = 0;
    if (++p.unit < line.per_entry) return;
    p.unit = 0;
    do ++p.entry; while (line.tiles(p.entry) == 0);
}

}  // namespace pg

struct PagedDecodeArgs {
    sc_paged_cache cache;
    const void* q; sc_dtype dt; int32_t B, Hq, Hkv, d; const int32_t* lens;
    float scale; void* out; void* ws; int32_t* status;
};
bool paged_decode_mma_supported(const PagedDecodeArgs& a);
cudaError_t launch_paged_decode_mma(const PagedDecodeArgs& a, cudaStream_t st);
size_t paged_decode_mma_ws_bytes();
cudaError_t launch_paged_decode_generic(const PagedDecodeArgs& a, cudaStream_t st);
size_t paged_decode_generic_ws_bytes(int32_t d);

struct PagedAppendArgs {
    sc_paged_cache cache; sc_paged_rows rows;
    sc_dtype dt; int32_t B, Hq, Hkv, T, d; uint32_t flags; int32_t* status;
};
cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st);

struct PagedSelectArgs {
    sc_paged_cache cache;
    const void* q; sc_dtype dt; int32_t B, Hq, Hkv, d; const int32_t* lens;
    int32_t keep, n_first, n_last; int32_t* sel_table; int32_t* sel_len; int32_t* status;
};
cudaError_t launch_paged_select(const PagedSelectArgs& a, cudaStream_t st);

}  // namespace sc
