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
    __host__ __device__ __forceinline__ int tiles_of(int n) const { return n > 0 ? (int)((unsigned)(n - 1) / (unsigned)tile) + 1 : 0; }   // (n may be 2^31 - 1)
    __device__ __forceinline__ int tiles(int e) const { return tiles_of(len(e)); }
    // Positions on the line are 32-bit numbers, which the entry point sees to: several divisions lie on the way to the first load.
};
struct Place {              // a position on the line
    int entry, unit, tile;
    unsigned at;            // of the unit's first tile
};

// Length of the line.  All lanes of a warp call it.
__device__ __forceinline__ unsigned total_of(const Line& line, int lane) {
    unsigned sum = 0;
#pragma unroll 4
    for (int e = lane; e < line.entries; e += 32) sum += line.tiles(e);
    return __reduce_add_sync(kFull, sum) * line.per_entry;
}

// The place of tile `at` of the line (at < total).  All lanes of a warp call it.
__device__ __forceinline__ Place place_of(const Line& line, unsigned at, int lane) {
    unsigned before = 0;
    for (int e0 = 0;; e0 += 32) {
        const int nt = e0 + lane < line.entries ? line.tiles(e0 + lane) : 0;
        const unsigned mine = (unsigned)nt * line.per_entry, upto = before + warp_scan_add((int)mine, lane);
        const unsigned past = __ballot_sync(kFull, upto > at);
        if (past != 0) {
            const int src = __ffs(past) - 1;
            const unsigned start = __shfl_sync(kFull, upto - mine, src), t = __shfl_sync(kFull, nt, src);
            Place p;
            p.entry = e0 + src;
            p.unit = (at - start) / t;
            p.at = start + p.unit * t;
            p.tile = at - p.at;
            return p;
        }
        before = __shfl_sync(kFull, upto, 31);
    }
}

// A line whose stretches would be short is cut at the units' ends instead, so that a party has one segment and fills its pipeline once:
// every unit in as many equal parts as have `longest` tiles at most, `longest` the least for which there are parties enough (at most an
// eighth over it).  For at most 64 entries and no more units than parties.  All lanes of a warp call it.
struct Part { int entry, unit, tile, take, index, parts; };   // take 0: this party has none
__device__ __forceinline__ Part part_of(const Line& line, unsigned longest, unsigned party, int lane) {
    const unsigned t0 = lane < line.entries ? line.tiles(lane) : 0, t1 = lane + 32 < line.entries ? line.tiles(lane + 32) : 0;
    unsigned c0, c1, sum;
    for (;; longest += longest / 8 + 1) {
        c0 = (t0 + longest - 1) / longest; c1 = (t1 + longest - 1) / longest;
        sum = __reduce_add_sync(kFull, c0 + c1) * line.per_entry;
        if (sum <= (unsigned)line.parties) break;
    }
    Part r = {0, 0, 0, 0, 0, 0};
    if (party >= sum) return r;
    const unsigned m0 = c0 * line.per_entry, u0 = warp_scan_add((int)m0, lane), all0 = __shfl_sync(kFull, u0, 31);
    const unsigned m1 = c1 * line.per_entry, u1 = all0 + warp_scan_add((int)m1, lane);
    const bool second = party >= all0;
    const int src = __ffs(__ballot_sync(kFull, (second ? u1 : u0) > party)) - 1;
    const unsigned start = __shfl_sync(kFull, second ? u1 - m1 : u0 - m0, src), parts = __shfl_sync(kFull, second ? c1 : c0, src);
    const unsigned nt = __shfl_sync(kFull, second ? t1 : t0, src), each = (nt + parts - 1) / parts;
    r.entry = src + (second ? 32 : 0);
    r.unit = (party - start) / parts;
    r.index = (party - start) - r.unit * parts;
    r.parts = parts;
    r.tile = r.index * each;
    r.take = min(each, nt - r.tile);   // ((parts - 1) * each < nt)
    return r;
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
