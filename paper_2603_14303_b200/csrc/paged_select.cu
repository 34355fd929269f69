// sc_paged_select: the pages that sparse attention reads.
//
// One cluster of blocks serves one (sequence, KV head); block r holds the r-th part of its pages.  Bounds are summed in 64 bits, turned
// into integers of the same order, and kept in shared memory; the keep-th largest is found digit by digit, each digit from a
// histogram over all pages of the head that the blocks add up through distributed shared memory.  A page's place in the result is
// the number of picked pages before it.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace sc {
namespace pg {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kMaxD = 256;
constexpr int kMaxGroupSmem = 64;   // query heads held at a time

// Integers in the order of the numbers; not-a-number above all.
__device__ __forceinline__ uint64_t key_of(double x) {
    if (x != x) return 0xfffffffffffffffeull;
    const int64_t i = __double_as_longlong(x + 0.0);   // (-0 is 0)
    return i < 0 ? ~(uint64_t)i : (uint64_t)i | 0x8000000000000000ull;
}
constexpr uint64_t kForced = 0xffffffffffffffffull;   // always picked
constexpr uint64_t kNoPage = 0ull;                    // a table entry that names none

template <typename T>
__global__ void __launch_bounds__(kThreads)
select_pages(const Pages<T> pages, const T* __restrict__ q, int Hq, int Hkv, int d, const int32_t* __restrict__ lens, int keep, int n_first, int n_last,
             int per_block, int32_t* __restrict__ sel_table, int32_t* __restrict__ sel_len, int32_t* status) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint64_t* keys = reinterpret_cast<uint64_t*>(smem);                     // [per_block]
    float* sq = reinterpret_cast<float*>(smem + (size_t)per_block * 8);     // [G][d]
    __shared__ int hist[256], total[256];
    __shared__ int sh_digit, sh_above, sh_greater, sh_equal, warp_n[kThreads / 32];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bh = blockIdx.x / C, b = bh / Hkv, h = bh - b * Hkv, G = Hq / Hkv, ps = pages.page_size;
    in_stream_order();
    const int entry = pages.table_heads > 1 ? bh : b;
    const int len = max(min(lens[entry], pages.cap()), 0), n = (len + ps - 1) / ps;
    const int32_t* table = pages.table_of(entry);
    int32_t* out = sel_table + (int64_t)bh * keep;
    if (n <= keep) {   // all of them
        for (int i = rank * kThreads + tid; i < keep; i += C * kThreads) out[i] = i < n ? table[i] : -1;
        if (rank == 0 && tid == 0) sel_len[bh] = len;
        return;
    }
    if (rank == 0 && tid == 0) sel_len[bh] = len - (n - keep) * ps;
    const int each = (n + C - 1) / C, p0 = min(rank * each, n), p1 = min(p0 + each, n);
    for (int i = tid; i < G * d; i += kThreads) sq[i] = Elem<T>::load(q + ((int64_t)b * Hq + h * G) * d + i);
    __syncthreads();
    const int hp = pages.page_heads > 1 ? h : 0;
    for (int p = p0 + warp; p < p1; p += kThreads / 32) {
        uint64_t key = kForced;
        if (p >= n_first && p < n - n_last) {
            const int id = table[p];
            key = kNoPage;
            if (pages.names_page(id)) {
                const T* mn = pages.k_min + ((int64_t)id * pages.page_heads + hp) * d;
                const T* mx = pages.k_max + ((int64_t)id * pages.page_heads + hp) * d;
                for (int g = 0; g < G; ++g) {
                    double s = 0.0;
                    for (int c = lane; c < d; c += 32) {
                        const double x = sq[g * d + c], lo = x * Elem<T>::load(mn + c), hi = x * Elem<T>::load(mx + c);
                        s += lo > hi || lo != lo ? lo : hi;
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
                    const uint64_t k = key_of(s);
                    key = k > key ? k : key;
                }
            } else if (lane == 0) {
                set_status(status, SC_ERR_INVALID_ARG);
            }
        }
        if (lane == 0) keys[p - p0] = key;
    }
    const int mine = p1 - p0;
    // the keep-th largest key: `want` pages still to come from those that agree with `prefix` in the digits so far
    uint64_t prefix = 0;
    int want = keep;
    for (int shift = 56; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < mine; i += kThreads)
            if (shift == 56 || keys[i] >> (shift + 8) == prefix) atomicAdd(&hist[(int)(keys[i] >> shift & 255)], 1);
        cluster.sync();
        int sum = 0;
        for (int r = 0; r < C; ++r) sum += cluster.map_shared_rank(hist, r)[tid];
        total[tid] = sum;
        cluster.sync();   // (the histograms may be cleared)
        if (tid == 0) {
            int above = 0, dg = 255;
            while (above + total[dg] < want) above += total[dg--];
            sh_digit = dg; sh_above = above;
        }
        __syncthreads();
        prefix = prefix << 8 | (uint64_t)sh_digit;
        want -= sh_above;
    }
    // this block's picked pages, and those with the last key: how many come from the blocks before
    if (tid == 0) { sh_greater = 0; sh_equal = 0; }
    __syncthreads();
    int greater = 0, equal = 0;
    for (int i = tid; i < mine; i += kThreads) { greater += keys[i] > prefix; equal += keys[i] == prefix; }
    atomicAdd(&sh_greater, greater);
    atomicAdd(&sh_equal, equal);
    cluster.sync();
    int before_greater = 0, before_equal = 0;
    for (int r = 0; r < rank; ++r) { before_greater += *cluster.map_shared_rank(&sh_greater, r); before_equal += *cluster.map_shared_rank(&sh_equal, r); }
    cluster.sync();
    for (int i0 = 0; i0 < mine; i0 += kThreads) {
        const int i = i0 + tid;
        const int g = i < mine && keys[i] > prefix, e = i < mine && keys[i] == prefix;
        const unsigned gb = __ballot_sync(kFull, g), eb = __ballot_sync(kFull, e);
        if (lane == 0) warp_n[warp] = __popc(gb) | __popc(eb) << 16;
        __syncthreads();
        int ng = 0, ne = 0, all_g = 0, all_e = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            const int x = warp_n[w];
            if (w < warp) { ng += x & 0xffff; ne += x >> 16; }
            all_g += x & 0xffff; all_e += x >> 16;
        }
        ng += before_greater + __popc(gb & ((1u << lane) - 1));
        ne += before_equal + __popc(eb & ((1u << lane) - 1));
        if (g || (e && ne < want)) out[ng + min(ne, want)] = table[p0 + i];
        before_greater += all_g; before_equal += all_e;
        __syncthreads();
    }
}

template <typename T>
cudaError_t run(const PagedSelectArgs& a, cudaStream_t st) {
    const Pages<T> pages = pages_of<T>(a.cache);
    const int64_t heads = (int64_t)a.B * a.Hkv;
    int C = 1;
    while (C < 16 && (a.cache.max_pages > 512 * C)) C *= 2;
    if (heads * C > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const int per_block = div_up(a.cache.max_pages, C);
    const size_t bytes = (size_t)per_block * 8 + sizeof(float) * (a.Hq / a.Hkv) * a.d;
    const auto kernel = select_pages<T>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return own_error(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(heads * C));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return own_error(cudaLaunchKernelEx(&cfg, kernel, pages, (const T*)a.q, a.Hq, a.Hkv, a.d, a.lens, a.keep, a.n_first, a.n_last, per_block, a.sel_table,
                                        a.sel_len, a.status));
}

}  // namespace

}  // namespace pg

cudaError_t launch_paged_select(const PagedSelectArgs& a, cudaStream_t st) {
    const cudaError_t e = a.dt == SC_BF16 ? pg::run<__nv_bfloat16>(a, st) : pg::run<float>(a, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
