// sc_paged_select: the pages that sparse attention reads.
//
// One cluster of blocks serves one (sequence, KV head); its block r scores the r-th part of the pages.
//   1. Bounds in fp32.  max(q m, q M) is q+ M + q- m, q+ and q- the query's positive and negative parts: with all pages' smallest and largest
//      keys side by side a matrix product against [q-; q+].  bf16: on the tensor cores (mma.m16n8k16, pages on M, eight queries on N).  fp32: a
//      lane has a page to itself, so that sums need no exchange between lanes.  Either way 64 bytes at a time of 32 pages' smallest and largest
//      keys come through a ring of cp.async stages per warp (chunks XOR-swizzled: rows of 128 bytes are read without conflicts).
//   2. The keep-th largest, T, of them, by the cluster's first block: a histogram between the smallest and the largest one, whose bin
//      that holds T has few keys as a rule; they are ranked one against the other.
//   3. What the fp32 sums are off by at most, delta, is known: so many roundings of sums no larger than the sum of |q_c| |bound_c|.  A page
//      above T + 2 delta is in, one below T - 2 delta is out, whatever 64 bits would say.  Those between are the keep-th itself and as a rule
//      none or two others; where they are more than there are places, they are scored again in 64 bits and their order decides, equal
//      ones by position: a few by the first block, many (pages that are all alike, or bounds that are not finite: delta is not either, then,
//      and all pages are between) by the cluster.
//   4. A page's place in the result is the number of picked pages before it.
#include <cooperative_groups.h>

#include <mutex>

#include "paged.cuh"
#include "umma.cuh"

namespace sc {
namespace pg {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;       // two blocks per SM: clusters of 16 find room where a GPC has fewer SMs
constexpr int kWarps = kThreads / 32;
constexpr int kPiece = 64;          // bytes of a row that are staged at a time
constexpr int kStageBytes = 32 * 2 * kPiece, kStages = 3;
constexpr int kRingBytes = kWarps * kStages * kStageBytes;
constexpr int kMaxCluster = 16;
constexpr int kGather = 16384;      // pages whose keys the first block copies to its own shared memory
constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr int kMaxSmem = 212 * 1024;   // dynamic, per block
constexpr int kFew = 128;           // keys, or pages between T - 2 delta and T + 2 delta, that the first block ranks one against the other
static_assert(kRingBytes + 8 * 2 * 256 * 4 + SC_SELECT_MAX_PAGES / kMaxCluster * 4 + 64 <= kMaxSmem &&
              kBins * 4 + SC_SELECT_MAX_PAGES / kMaxCluster * 12 + 8 * 2 * 256 * 4 + 64 <= kMaxSmem, "");
static_assert(kBins % kThreads == 0 && kFew <= kThreads, "");

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

// 32-bit keys in the order of the numbers.  Always picked: the largest one; a table entry that names no page: 0, below all numbers.
constexpr uint32_t kForced = 0xffffffffu, kNoPage = 0u;
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);   // (-0 is 0)
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
// 64-bit ones; not-a-number above all numbers.
__device__ __forceinline__ uint64_t key_of(double x) {
    if (x != x) return ~0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

constexpr uint32_t kNaN = 0x7fffffffu;   // (and the mask of a magnitude: the order of such integers is that of the magnitudes, NaN above infinity)
__device__ __forceinline__ uint32_t largest_of(const float4& w) {
    return max(max(__float_as_uint(w.x) & kNaN, __float_as_uint(w.y) & kNaN), max(__float_as_uint(w.z) & kNaN, __float_as_uint(w.w) & kNaN));
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

struct Verdict {           // of the first block, for the cluster
    uint32_t lo, hi;       // keys in [lo, hi] are between; larger ones are in
    int many;              // the cluster scores those again in 64 bits
};

struct Sizes { int ring, gather; };   // of the shared memory's first part in bytes, of the first block's array of keys (even)

template <typename T> struct Path;
template <> struct Path<__nv_bfloat16> { static constexpr int kG = 8; };   // query heads at a time; with more the pages go by again
template <> struct Path<float> { static constexpr int kG = 4; };

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
select_pages(const Pages<const T> pages, const T* __restrict__ q, int Hq, int Hkv, int d, const int32_t* __restrict__ lens, int keep, int n_first, int n_last,
             const Sizes sizes, int32_t* __restrict__ sel_table, int32_t* __restrict__ sel_len, int32_t* status) {
    constexpr bool kMma = sizeof(T) == 2;
    constexpr int E = 16 / sizeof(T), kCols = kPiece / sizeof(T), kG = Path<T>::kG;
    const int gather = sizes.gather;
    extern __shared__ __align__(128) unsigned char smem[];
    const int pieces = max((d + kCols - 1) / kCols, kStages - 1), wide = pieces * kCols;   // (the ring looks no further than the next pages)
    // [the ring, and in its place once the bounds are there: histogram, all pages' keys (the first block's), 64-bit keys of this block's
    // pages][queries: kG x positive and negative parts x columns, whole pieces (bf16: as the product's B operand, lane by lane)][keys of this
    // block's pages]
    int* hist = reinterpret_cast<int*>(smem);                                           // [kBins]
    uint32_t* gathered = reinterpret_cast<uint32_t*>(hist + kBins);                     // [gather]
    uint64_t* keys64 = reinterpret_cast<uint64_t*>(gathered + gather);                  // [per_block], of the pages between
    float* sq = reinterpret_cast<float*>(smem + sizes.ring);
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem + sizes.ring + kG * 2 * wide * sizeof(T));   // [per_block]
    __shared__ uint32_t sh_largest, sh_low, sh_high;   // bits of the largest sum of |q_c| |bound_c| (fp32: of the largest |bound|); smallest and
                                                   // largest key of a number
    __shared__ float sh_norm;                      // fp32: largest 1-norm of a query
    __shared__ Verdict sh_verdict;
    __shared__ int2 sh_warp[2][kWarps];
    __shared__ int sh_bin, sh_bin_above, sh_bin_n, sh_few;
    __shared__ int few_page[kFew];                 // pages between, and whether they are in
    __shared__ uint64_t few_key[kFew];
    __shared__ bool few_in[kFew];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bh = blockIdx.x / C, b = bh / Hkv, h = bh - b * Hkv, G = Hq / Hkv, ps = pages.page_size;
    if (tid == 0) { sh_largest = 0; sh_low = kForced; sh_high = 0; sh_norm = kMma ? 1.f : 0.f; sh_few = 0; sh_bin_n = 0; }
    in_stream_order();
    const int entry = pages.table_heads > 1 ? bh : b;
    const int len = max(min(lens[entry], pages.cap()), 0), n = len > 0 ? (len - 1) / ps + 1 : 0;
    const int32_t* table = pages.table_of(entry);
    int32_t* out = sel_table + (int64_t)bh * keep;
    if (n <= keep) {   // all of them
        for (int i = rank * kThreads + tid; i < keep; i += C * kThreads) out[i] = i < n ? table[i] : -1;
        if (rank == 0 && tid == 0) sel_len[bh] = len;
        return;
    }
    if (rank == 0 && tid == 0) sel_len[bh] = len - (n - keep) * ps;
    __syncthreads();
    const int each = ((n + C - 1) / C + 3) & ~3, p0 = min(rank * each, n), p1 = min(p0 + each, n);
    const int hp = pages.page_heads > 1 ? h : 0;
    const T* qh = q + ((int64_t)b * Hq + h * G) * d;
    const bool local = C == 1 || n <= gather;   // the first block has the keys of all pages in its own shared memory
    const auto forced = [&](int p) { return p < n_first || p >= n - n_last; };
    // A page's bound in 64 bits, by a warp; a table entry that names no page: 0.  The page is read once for four queries (8 heads x 8192 pages
    // 26.8 us with once per query, 26.0), with one or two for each (zeros in the others' places: 11.6 against 12.0).
    const auto score_for = [&](int64_t at, int g0, auto& s) {
        constexpr int kN = sizeof(s) / sizeof(s[0]);
#pragma unroll 2
        for (int c = lane; c < d; c += 32) {
            const double low = Elem<T>::load(pages.k_min + at + c), high = Elem<T>::load(pages.k_max + at + c);
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                const double x = g0 + j < G ? Elem<T>::load(qh + (int64_t)(g0 + j) * d + c) : 0.f, y = x * low, z = x * high;
                s[j] += y > z || y != y ? y : z;
            }
        }
        uint64_t best = 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int j = 0; j < kN; ++j) s[j] += __shfl_xor_sync(kFull, s[j], o);
#pragma unroll
        for (int j = 0; j < kN; ++j)
            if (g0 + j < G && key_of(s[j]) > best) best = key_of(s[j]);
        return best;
    };
    const auto score64 = [&](int p, uint32_t k) {
        uint64_t best = 0;
        if (k == kNoPage) return best;
        const int64_t at = ((int64_t)table[p] * pages.page_heads + hp) * d;
        for (int g0 = 0; g0 < G; g0 += G > 2 ? 4 : 1) {
            double four[4] = {0.0, 0.0, 0.0, 0.0}, one[1] = {0.0};
            const uint64_t x = G > 2 ? score_for(at, g0, four) : score_for(at, g0, one);
            if (x > best) best = x;
        }
        return best;
    };

    // ---- 1: bounds in fp32 ----
    {
        const auto entry_at = [&](int p) { return p < p1 && !forced(p) ? table[p] : -1; };
        const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (kStages * kStageBytes);
        // Piece `at` of the pages `ids` (lane l has the l-th): four lanes copy a page's 64 bytes of smallest keys, then of largest ones.
        const auto copy = [&](int stage, int ids, int at) {
            const int c = lane & 3, col = at * kCols + c * E;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2), id = __shfl_sync(kFull, ids, r);
                const bool ok = pages.names_page(id) && col < d;
                const int64_t o = ((int64_t)id * pages.page_heads + hp) * d + col;
                const uint32_t row = ring + stage * kStageBytes + r * (2 * kPiece);
                cp_async16(row + ((c ^ (r & 7)) << 4), ok ? (const void*)(pages.k_min + o) : q, ok ? 16 : 0);
                cp_async16(row + (((c + 4) ^ (r & 7)) << 4), ok ? (const void*)(pages.k_max + o) : q, ok ? 16 : 0);
            }
        };
        uint32_t largest = 0, low = kForced, high = 0;
        for (int g0 = 0; g0 < G; g0 += kG) {
            if (g0 > 0) __syncthreads();
            for (int i = tid; i < kG * wide; i += kThreads) {
                const int g = i / wide, c = i - g * wide;
                const float x = g0 + g < G && c < d ? Elem<T>::load(qh + (int64_t)(g0 + g) * d + c) : 0.f;
                const float up = x > 0.f || x != x ? x : 0.f, down = x < 0.f || x != x ? x : 0.f;
                if constexpr (kMma) {
                    // B of step c / 16: lane (g, (c % 8) / 2) has columns c % 16 and, in its second register, those eight further on
                    T* to = reinterpret_cast<T*>(sq) + ((c / 16 * 2 * 32 + g * 4 + c % 8 / 2) * 4 + c % 16 / 8 * 2 + c % 2);
                    Elem<T>::store(to, down);
                    Elem<T>::store(to + 32 * 4, up);
                } else {
                    sq[g * 2 * wide + c] = up;
                    sq[g * 2 * wide + wide + c] = down;
                }
            }
            // the ring runs kStages - 1 pieces ahead, into the next pages (`then`: which of them)
            int base = p0 + warp * 32, ids = entry_at(base + lane), next_ids = entry_at(base + kWarps * 32 + lane), stage = 0, ahead = 0, then = 0;
            const auto request = [&](int to, int here) {     // the next piece, if there is one
                if (ahead < pieces) {
                    if (here < p1) copy(to, ids, ahead);
                    ++ahead;
                } else {
                    if (here + kWarps * 32 < p1 && then < pieces) copy(to, next_ids, then);
                    ++then;
                }
                cp_async_commit();
            };
#pragma unroll
            for (int i = 0; i < kStages - 1; ++i) request(i, base);
            __syncthreads();   // (the queries)
            for (; base < p1; base += kWarps * 32) {
                const int p = base + lane;
                if (p < p1 && !forced(p) && !pages.names_page(ids)) set_status(status, SC_ERR_INVALID_ARG);
                // fp32: a lane's page, per query, two halves of the columns.  bf16: C of two products of 16 pages, and of the products of magnitudes
                float2 acc[kMma ? 1 : kG];
                float cs[2][4], cm[2][4];
#pragma unroll
                for (int g = 0; g < (kMma ? 1 : kG); ++g) acc[g] = make_float2(0.f, 0.f);
#pragma unroll
                for (int m = 0; m < 2; ++m) cs[m][0] = cs[m][1] = cs[m][2] = cs[m][3] = cm[m][0] = cm[m][1] = cm[m][2] = cm[m][3] = 0.f;
                for (int at = 0; at < pieces; ++at, stage = stage + 1 == kStages ? 0 : stage + 1) {
                    request(stage == 0 ? kStages - 1 : stage - 1, base);
                    cp_async_wait<kStages - 1>();
                    __syncwarp();
                    if constexpr (kMma) {
                        const uint32_t rows = ring + stage * kStageBytes;
                        const int lm_j = lane >> 3, lm_r = (lane & 7) + ((lm_j & 1) << 3);   // matrices (rows 0-7, 8-15) x (chunk, the next)
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const uint2* bq = reinterpret_cast<const uint2*>(sq) + (at * 2 + s) * 64 + lane;
                            const uint2 down = bq[0], up = bq[32];
                            const uint2 mag = make_uint2(up.x | (down.x & 0x7fff7fffu), up.y | (down.y & 0x7fff7fffu));
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const int c = 2 * s + (lm_j >> 1);
                                const uint32_t row = rows + (m * 16 + lm_r) * (2 * kPiece);
                                uint32_t a[4], z[4];
                                ldmatrix_x4(row + ((c ^ (lm_r & 7)) << 4), a);
                                ldmatrix_x4(row + (((c + 4) ^ (lm_r & 7)) << 4), z);
                                mma_bf16(cs[m], a, down.x, down.y);
                                mma_bf16(cs[m], z, up.x, up.y);
#pragma unroll
                                for (int i = 0; i < 4; ++i) a[i] = __vmaxu2(a[i] & 0x7fff7fffu, z[i] & 0x7fff7fffu);
                                mma_bf16(cm[m], a, mag.x, mag.y);
                            }
                        }
                    } else {
                        float2 part[kG];      // (sums of a piece by themselves: shorter chains of roundings)
#pragma unroll
                        for (int g = 0; g < kG; ++g) part[g] = make_float2(0.f, 0.f);
                        const unsigned char* row = smem + warp * (kStages * kStageBytes) + stage * kStageBytes + lane * (2 * kPiece);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float4 a = *reinterpret_cast<const float4*>(row + ((c ^ (lane & 7)) << 4));
                            const float4 z = *reinterpret_cast<const float4*>(row + (((c + 4) ^ (lane & 7)) << 4));
                            largest = max(largest, max(largest_of(a), largest_of(z)));
                            const float* up = sq + at * kCols + c * E;
#pragma unroll
                            for (int g = 0; g < kG; ++g, up += 2 * wide) {
                                const float4 u = *reinterpret_cast<const float4*>(up), w = *reinterpret_cast<const float4*>(up + wide);
                                part[g] = umma::fma2(make_float2(u.x, u.y), make_float2(z.x, z.y), umma::fma2(make_float2(w.x, w.y), make_float2(a.x, a.y), part[g]));
                                part[g] = umma::fma2(make_float2(u.z, u.w), make_float2(z.z, z.w), umma::fma2(make_float2(w.z, w.w), make_float2(a.z, a.w), part[g]));
                            }
                        }
#pragma unroll
                        for (int g = 0; g < kG; ++g) { acc[g].x += part[g].x; acc[g].y += part[g].y; }
                    }
                    __syncwarp();   // (the stage is written again)
                }
                float best = -INFINITY;
                int l = lane;                 // the page, among the 32, that this lane ends up with
                if constexpr (kMma) {
                    const int tig = lane & 3;
                    float of[4];              // pages lane / 4 + 0, 8, 16, 24
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool one = g0 + 2 * tig < G, two = g0 + 2 * tig + 1 < G;
                        const float x = cs[i >> 1][i % 2 * 2], y = cs[i >> 1][i % 2 * 2 + 1];
                        of[i] = fmaxf(one ? x : -INFINITY, two ? y : -INFINITY);
                        of[i] = fmaxf(of[i], __shfl_xor_sync(kFull, of[i], 1));
                        of[i] = fmaxf(of[i], __shfl_xor_sync(kFull, of[i], 2));
                        if (one) largest = max(largest, __float_as_uint(cm[i >> 1][i % 2 * 2]) & kNaN);
                        if (two) largest = max(largest, __float_as_uint(cm[i >> 1][i % 2 * 2 + 1]) & kNaN);
                    }
                    best = tig == 0 ? of[0] : tig == 1 ? of[1] : tig == 2 ? of[2] : of[3];
                    l = tig * 8 + (lane >> 2);
                } else {
#pragma unroll
                    for (int g = 0; g < kG; ++g)
                        if (g0 + g < G) best = fmaxf(best, acc[g].x + acc[g].y);
                }
                const int my_id = __shfl_sync(kFull, ids, l), mp = base + l;
                if (mp < p1) {
                    const bool counts = !forced(mp) && pages.names_page(my_id);
                    uint32_t k = min(max(key_of(best), kNoPage + 1), kForced - 1);   // (only what is not finite has such keys)
                    if (g0 > 0) k = max(k, keys[mp - p0]);
                    if (!counts) k = forced(mp) ? kForced : kNoPage;
                    keys[mp - p0] = k;
                    if (g0 + kG >= G && counts) { low = min(low, k); high = max(high, k); }
                }
                ids = next_ids;
                next_ids = entry_at(base + 2 * kWarps * 32 + lane);
                ahead = then; then = 0;
            }
            cp_async_wait<0>();
        }
        largest = __reduce_max_sync(kFull, largest);
        low = __reduce_min_sync(kFull, low);
        high = __reduce_max_sync(kFull, high);
        if (lane == 0) { atomicMax(&sh_largest, largest); atomicMin(&sh_low, low); atomicMax(&sh_high, high); }
    }
    if (!kMma && rank == 0) {
        for (int g = warp; g < G; g += kWarps) {
            float s = 0.f;
            for (int c = lane; c < d; c += 32) s += fabsf(Elem<T>::load(qh + (int64_t)g * d + c));
            s = warp_sum(s);
            if (lane == 0) atomicMax(reinterpret_cast<unsigned*>(&sh_norm), s == s ? __float_as_uint(s) : kNaN);
        }
    }
    cluster.sync();

    // ---- 2 and 3: the first block finds what is in, what is out, and whether the rest needs 64 bits ----
    const auto remote32 = [&](int p) { const int r = p / each; return cluster.map_shared_rank(keys, r)[p - r * each]; };
    const auto remote64 = [&](int p) { const int r = p / each; return cluster.map_shared_rank(keys64, r)[p - r * each]; };
    const uint32_t* near = C == 1 ? keys : gathered;
    const auto key_at = [&](int p) { return local ? near[p] : remote32(p); };
    const auto set_key = [&](int p, uint32_t k) {
        if (local) { const_cast<uint32_t*>(near)[p] = k; } else { const int r = p / each; cluster.map_shared_rank(keys, r)[p - r * each] = k; }
    };
    const auto for_keys = [&](auto&& f) {         // all pages' keys, shared out among the threads
        if (local) {
            for (int v = tid; v < (n + 3) / 4; v += kThreads) {
                const uint4 k = reinterpret_cast<const uint4*>(near)[v];
                f(4 * v, k.x);
                if (4 * v + 1 < n) f(4 * v + 1, k.y);
                if (4 * v + 2 < n) f(4 * v + 2, k.z);
                if (4 * v + 3 < n) f(4 * v + 3, k.w);
            }
        } else {
            for (int p = tid; p < n; p += kThreads) f(p, remote32(p));
        }
    };
    int turn = 0;
    const auto block_sums = [&](int x, int y) {   // over all threads
        x = __reduce_add_sync(kFull, x); y = __reduce_add_sync(kFull, y);
        int2* w = sh_warp[turn ^= 1];             // (two places by turns: one barrier per sum)
        if (lane == 0) w[warp] = make_int2(x, y);
        __syncthreads();
        const int2 t = lane < kWarps ? w[lane] : make_int2(0, 0);
        return make_int2(__reduce_add_sync(kFull, t.x), __reduce_add_sync(kFull, t.y));
    };
    const auto warps_before = [&] {               // the last sums' parts from the warps before this one
        int2 t = make_int2(0, 0);
        for (int i = 0; i < warp; ++i) { t.x += sh_warp[turn][i].x; t.y += sh_warp[turn][i].y; }
        return t;
    };
    // Warp w has the pages [r0, r1), w * run on, where their order counts.
    const int run = (n + kWarps - 1) / kWarps, r0 = min(warp * run, n), r1 = min(r0 + run, n);
    int above = 0;     // pages that are in without question
    uint32_t first_in = 0;                        // keys from here on are in
    int2 before = make_int2(0, 0);                // pages in, and ties, of the warps before
    if (rank == 0) {
        const int from = lane < C ? lane : 0;
        const uint32_t largest = __reduce_max_sync(kFull, *cluster.map_shared_rank(&sh_largest, from));
        const uint32_t low = __reduce_min_sync(kFull, *cluster.map_shared_rank(&sh_low, from));
        const uint32_t high = __reduce_max_sync(kFull, *cluster.map_shared_rank(&sh_high, from));
        // bins of 2^shift keys from the smallest on; bin 0 also has what names no page, and what is always picked lies above all bins
        const int spread = low < high ? 32 - __clz(high - low) : 0, shift = max(spread - kBinBits, 0);
        const auto bin_of = [&](uint32_t k) { return k <= low ? 0 : (int)((k - low) >> shift); };
        for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        if (local && C > 1) {
            const unsigned each4 = each / 4, n4 = (n + 3) / 4;     // (each block's part is a multiple of four)
#pragma unroll 1
            for (unsigned v0 = tid; v0 < n4; v0 += 8 * kThreads) {
                uint4 k[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const unsigned v = min(v0 + j * kThreads, n4 - 1), r = v / each4;
                    k[j] = reinterpret_cast<const uint4*>(cluster.map_shared_rank(keys, r))[v - r * each4];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (v0 + j * kThreads < n4) reinterpret_cast<uint4*>(gathered)[v0 + j * kThreads] = k[j];
            }
            __syncthreads();
        }
        int over = 0;
        for_keys([&](int, uint32_t k) {
            if (k == kForced) ++over; else atomicAdd(&hist[bin_of(k)], 1);
        });
        over = block_sums(over, 0).x;
        uint32_t kth = kForced;
        if (over < keep && low > high) {
            kth = kNoPage;                    // nothing names a page
        } else if (over < keep) {
            // the bin of the keep-th largest: thread t has bins [t * 8, t * 8 + 8) from above
            constexpr int kMine = kBins / kThreads;
            int mine = 0;
#pragma unroll
            for (int i = 0; i < kMine; ++i) mine += hist[kBins - 1 - (tid * kMine + i)];
            int upto = warp_scan_add(mine, lane);
            int2* w = sh_warp[turn ^= 1];
            if (lane == 31) w[warp].x = upto;
            __syncthreads();
            for (int i = 0; i < warp; ++i) upto += w[i].x;
            upto += over;
            if (upto >= keep && upto - mine < keep) {
                int bin = kBins - 1 - tid * kMine, sum = upto - mine;
                while (sum + hist[bin] < keep) sum += hist[bin--];
                sh_bin = bin; sh_bin_above = sum;
            }
            __syncthreads();
            const int bin = sh_bin, want = keep - sh_bin_above, in_bin = hist[bin];
            if (in_bin <= kFew) {
                for_keys([&](int, uint32_t k) {
                    if (k != kForced && bin_of(k) == bin) few_key[atomicAdd(&sh_bin_n, 1)] = k;   // (any order)
                });
                __syncthreads();
                if (tid < in_bin) {           // the key that fewer than `want` are larger than, but not fewer than `want` as large
                    const uint64_t k = few_key[tid];
                    int larger = 0, equal = 0;
                    for (int j = 0; j < in_bin; ++j) { larger += few_key[j] > k; equal += few_key[j] == k; }
                    if (larger < want && larger + equal >= want) sh_bin = (int)(uint32_t)k;   // (equal ones write the same)
                }
                __syncthreads();
                kth = (uint32_t)sh_bin;
            } else {                          // bit by bit
                kth = 0;
                for (int bit = 31; bit >= 0; --bit) {
                    const uint32_t c = kth | 1u << bit;
                    int m = 0;
                    for_keys([&](int, uint32_t k) { m += k >= c; });
                    if (block_sums(m, 0).x >= keep) kth = c;
                }
            }
        }
        // fp32: a piece's products in a row, the pieces, and the two halves of the columns, rounded to nearest.  bf16: the products are exact; a
        // product's step adds 16 of them to the sum, in at least single precision but any order and rounding: what each addition drops is 2^-23
        // of the sum of magnitudes at most.  (1.01: the norms' and sums' own rounding.  At the end: terms too small for fp32.)
        const float unit = kMma ? (wide / 8 * 17) * 0x1p-23f : (kCols + pieces + 1) * 0x1p-24f;
        const float delta = unit * 1.01f * (sh_norm * __uint_as_float(largest)) + 0x1p-110f;
        uint32_t lo, hi;
        if (!(delta < INFINITY)) {
            lo = kNoPage; hi = kForced - 1;
        } else if (kth == kForced || kth == kNoPage) {
            lo = hi = kth;
        } else {
            const float t = value_of(kth);
            lo = max(key_of(__fadd_rd(t, -2.f * delta)), kNoPage + 1); hi = min(key_of(__fadd_ru(t, 2.f * delta)), kForced - 1);
        }
        int na = 0, nb = 0;
        for (int b0 = r0; b0 < r1; b0 += 4 * 32) {
            uint32_t k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = b0 + 32 * j + lane < r1 ? key_at(b0 + 32 * j + lane) : kNoPage;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int p = b0 + 32 * j + lane;
                na += p < r1 && k[j] > hi;
                if (p < r1 && k[j] >= lo && k[j] <= hi) {
                    ++nb;
                    const int i = atomicAdd(&sh_few, 1);     // (any order: what follows goes by page)
                    if (i < kFew) few_page[i] = p;
                }
            }
        }
        const int2 s = block_sums(na, nb);
        before = warps_before();
        above = s.x;
        const bool again = above + s.y != keep;
        if (tid < C) {   // (told to everybody here: nobody looks into this block's shared memory afterwards)
            Verdict* v = cluster.map_shared_rank(&sh_verdict, tid);
            v->lo = lo; v->hi = hi; v->many = again && s.y > kFew;
        }
        if (again && s.y <= kFew) {
            for (int j = warp; j < s.y; j += kWarps) {
                const uint64_t x = score64(few_page[j], key_at(few_page[j]));
                if (lane == 0) few_key[j] = x;
            }
            __syncthreads();
            if (tid < s.y) {                  // those that are in get the largest key; the others now lie below
                int better = 0;
                for (int j = 0; j < s.y; ++j) better += few_key[j] > few_key[tid] || (few_key[j] == few_key[tid] && few_page[j] < few_page[tid]);
                few_in[tid] = better < keep - above;
                if (few_in[tid]) set_key(few_page[tid], kForced);
            }
            __syncthreads();
            int more = 0;
            for (int j = lane; j < s.y; j += 32) more += few_in[j] && few_page[j] < r0;
            before = make_int2(before.x + __reduce_add_sync(kFull, more), 0);
            first_in = hi + 1;
        } else {
            before = make_int2(before.x + before.y, 0);
            first_in = lo;
        }
    }
    // Where the first block has all the keys it needs, the others have done their part when it says so.
    cluster.sync();
    const Verdict verdict = sh_verdict;
    uint64_t T64 = 0;
    int ties = keep;                  // pages with exactly T64 that are in
    if (verdict.many) {
        for (int p = p0 + warp; p < p1; p += kWarps) {
            const uint32_t k = keys[p - p0];
            if (k < verdict.lo || k > verdict.hi) continue;
            const uint64_t x = score64(p, k);
            if (lane == 0) keys64[p - p0] = x;
        }
        cluster.sync();
        if (rank == 0) {
            const int want = keep - above;
            int more = 0;             // pages between whose key is larger than T64
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t c = T64 | 1ull << bit;
                int m = 0;
                for_keys([&](int p, uint32_t k) {
                    if (k >= verdict.lo && k <= verdict.hi) m += remote64(p) >= c;
                });
                m = block_sums(m, 0).x;
                if (m >= want) T64 = c; else more = m;
            }
            ties = want - more;
        }
    }

    // ---- 4: picked pages in order ----
    if (rank == 0) {
        // their positions first, the table's entries for them then all at once
        int* place = keep <= kBins ? hist : out;
        const unsigned below = (1u << lane) - 1;
        if (!verdict.many) {
            for (int b0 = r0; b0 < r1; b0 += 4 * 32) {
                uint32_t k[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = b0 + 32 * j + lane < r1 ? key_at(b0 + 32 * j + lane) : kNoPage;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = b0 + 32 * j + lane < r1 && k[j] >= first_in;
                    const unsigned ins = __ballot_sync(kFull, in);
                    if (in) place[before.x + __popc(ins & below)] = b0 + 32 * j + lane;
                    before.x += __popc(ins);
                }
            }
        } else {
            const auto look = [&](int p, int& in, int& tie) {
                const uint32_t k = key_at(p);
                in = k > verdict.hi; tie = 0;
                if (!in && k >= verdict.lo) {
                    const uint64_t x = remote64(p);
                    in = x > T64; tie = x == T64;
                }
            };
            int2 mine = make_int2(0, 0);
            for (int p = r0 + lane; p < r1; p += 32) { int in, tie; look(p, in, tie); mine.x += in; mine.y += tie; }
            block_sums(mine.x, mine.y);
            before = warps_before();
            for (int b0 = r0; b0 < r1; b0 += 32) {
                int in = 0, tie = 0;
                if (b0 + lane < r1) look(b0 + lane, in, tie);
                const unsigned ins = __ballot_sync(kFull, in), eqs = __ballot_sync(kFull, tie);
                const int eq = before.y + __popc(eqs & below);
                if (in || (tie && eq < ties)) place[before.x + __popc(ins & below) + min(eq, ties)] = b0 + lane;
                before.x += __popc(ins); before.y += __popc(eqs);
            }
        }
        __syncthreads();
        for (int i = tid; i < keep; i += kThreads) out[i] = table[place[i]];
    }
    if (!local || verdict.many) cluster.sync();   // (keys are read from here)
}

template <typename T>
cudaError_t start(const PagedSelectArgs& a, cudaStream_t st) {
    const auto kernel = select_pages<T>;
    const int64_t heads = (int64_t)a.B * a.Hkv;
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    static std::once_flag once[64];   // per device
    static cudaError_t ready[64];
    std::call_once(once[dev & 63], [&] {
        ready[dev & 63] = opt_in(kernel, kMaxSmem, true);
    });
    if (ready[dev & 63] != cudaSuccess) return ready[dev & 63];
    // As wide as leaves every block an SM, and 64 pages where the tables are full: 8 heads x 8192 pages in clusters of 16 27 us, of eight 28, of four 37; 32 heads
    // x 2048 pages in clusters of four 18, of two 21, of eight 20; 128 heads x 1024 pages single blocks 22, in twos 23.
    int C = 1;
    while (C < kMaxCluster && heads * C * 2 <= sms && a.cache.max_pages > 64 * C) C *= 2;
    while (C < kMaxCluster && a.cache.max_pages > 8192 * C) C *= 2;   // what a block has room for
    if (heads * C > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const int per_block = (div_up(a.cache.max_pages, C) + 3) / 4 * 4;
    const int cols = kPiece / (int)sizeof(T), pieces = div_up(a.d, cols) > kStages - 1 ? div_up(a.d, cols) : kStages - 1;
    const int rest = Path<T>::kG * 2 * pieces * kPiece + per_block * 4;
    Sizes sizes;
    const auto first_part = [&](int gather) {
        const int later = kBins * 4 + gather * 4 + per_block * 8;
        return later > kRingBytes ? (later + 15) / 16 * 16 : kRingBytes;
    };
    sizes.gather = C == 1 ? 0 : a.cache.max_pages < kGather ? (a.cache.max_pages + 3) / 4 * 4 : kGather;
    if (first_part(sizes.gather) + rest > kMaxSmem) sizes.gather = 0;
    sizes.ring = first_part(sizes.gather);
    const size_t bytes = (size_t)sizes.ring + rest;
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
    return own_error(cudaLaunchKernelEx(&cfg, kernel, pages_of<const T>(a.cache), (const T*)a.q, a.Hq, a.Hkv, a.d, a.lens, a.keep, a.n_first, a.n_last,
                                        sizes, a.sel_table, a.sel_len, a.status));
}

}  // namespace

}  // namespace pg

cudaError_t launch_paged_select(const PagedSelectArgs& a, cudaStream_t st) {
    const cudaError_t e = a.dt == SC_BF16 ? pg::start<__nv_bfloat16>(a, st) : pg::start<float>(a, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
