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
    int page_bits;                // page_size = 2^page_bits, or -1

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
    p.page_bits = -1;
    for (int i = 0; i < 31; ++i)
        if (c.page_size == 1 << i) p.page_bits = i;
    return p;
}

}  // namespace pg

namespace pg {

// The opt-ins of a kernel: its dynamic shared memory, and clusters beyond the portable size.
template <typename K>
inline cudaError_t opt_in(K kernel, int smem, bool wide) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && wide) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return own_error(e);
}

}  // namespace pg

struct PagedDecodeArgs {
    sc_paged_cache cache;
    const void* q; sc_dtype dt; int32_t B, Hq, Hkv, d; const int32_t* lens;
    float scale; void* out; void* ws; int32_t* status;
};
bool paged_decode_mma_supported(const PagedDecodeArgs& a);
cudaError_t launch_paged_decode_mma(const PagedDecodeArgs& a, cudaStream_t st);
size_t paged_decode_ws_bytes();
cudaError_t launch_paged_decode_generic(const PagedDecodeArgs& a, cudaStream_t st);

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
