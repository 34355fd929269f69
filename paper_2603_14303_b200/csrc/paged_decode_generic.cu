// sc_paged_decode_attn for any type and head size (d a multiple of 8 up to 256): the scores and the weighted sum on CUDA cores, in fp32.
//
// The frame is the tensor-core kernel's (paged_attn.cuh): a party takes a stretch of the line of 16-row tiles, a warp's tiles come through a ring
// of cp.async stages.  A row's 16-byte chunks lie XOR-swizzled in a place of a multiple of 128 bytes.  Scores: a lane has one of the 16
// rows and every other chunk of it (the queries are read by broadcast), so one exchange between lanes finishes a score.  Weighted sum: a lane has
// a chunk of columns (or two) and every row, or every R-th where a row has few chunks.  Bounded by its loads: a tile's two products take
// 650 instructions of a warp for 16 KB (float32, d = 128, four queries).
// Serves SC_F32 and head sizes that the tensor-core kernel does not take, and cross-checks it.
#include <mutex>

#include "paged_attn.cuh"

namespace sc {
namespace pg {

namespace {

constexpr float kMaxSlack = 8.f;          // log2 units a score may exceed the running maximum before it is raised

__device__ __forceinline__ void unpack(const uint4& w, float (&x)[8]) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(a[i] << 16); x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
}
__device__ __forceinline__ void unpack(const uint4& w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
}

__host__ __device__ inline int pitch_of(int d, int esize) { return (d * esize + 127) / 128 * 128; }
__host__ __device__ inline int stage_bytes(int pitch) { return 2 * kTile * pitch + 80; }   // K, V, 16 counts, which rows count

// What an SM holds at once hides the latency of the steps of one warp: three blocks, two with eight query heads, and a ring that leaves room for
// them (rows of 512 bytes: one stage, 16 sequences x 8 heads x 4 K rows of float32 108 us, with three stages and one block per SM 186).
__host__ __device__ constexpr int blocks_by_registers(int heads) { return heads <= 4 ? 3 : 2; }
__host__ __device__ constexpr int stages_of(int pitch) { return pitch <= 128 ? 3 : pitch <= 256 ? 2 : 1; }

// kH: query heads of a unit.  kStages: of a warp's ring.  kChunks: a lane's chunks of columns.
template <typename T, int kH, int kStages, int kChunks>
__global__ void __launch_bounds__(kThreads, blocks_by_registers(kH))
paged_decode_generic(const Pages<const T> pages, const T* __restrict__ q, int Hq, int Hkv, int d, Line line, const Division how, float scale_log2,
                     T* __restrict__ out, int32_t* __restrict__ tickets, float* __restrict__ part, int32_t* status) {
    constexpr int E = 16 / sizeof(T);
    extern __shared__ __align__(128) unsigned char smem[];
    const int pitch = pitch_of(d, sizeof(T)), stage_size = stage_bytes(pitch), ring_size = kWarps * kStages * stage_size;
    float* sq = reinterpret_cast<float*>(smem + ring_size);                             // queries [kH][d]
    __shared__ __align__(16) float sp[kWarps][kTile][kH];                              // weights of a tile
    __shared__ float sh_m[kWarps][kHeads], sh_l[kWarps][kHeads];
    __shared__ int sh_last;
    __shared__ __align__(8) unsigned long long sh_bar[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Party me;
    me.set_up(sh_bar);
    in_stream_order();
    const int G = Hq / Hkv;
    if (!me.plan(line, how, lane)) {
        zero_empty(pages, line, Hq, G, kH, d, out);
        me.step();
        return;
    }
    Joiner joiner = {sh_bar, smem + ring_size + kH * d * 4, &sh_last, tickets, part, status, kH, 0u, true};
    const int chunks = d / E;                            // of a row
    int width = 2;                                       // lanes that a row's chunks are spread over (a tile has 16 rows)
    while (width < chunks && width < 32) width *= 2;
    const int c0 = lane % width, v0 = lane / width, step = 32 / width;
    const uint32_t ring = smem_u32(smem) + warp * (kStages * stage_size);
    const unsigned char* ring_p = smem + warp * (kStages * stage_size);

    for (Place p = me.begin(line, lane);;) {
        const int len = line.len(p.entry), nt = line.tiles(p.entry);
        const int take = (int)min((unsigned)(nt - p.tile), me.left);
        const Unit unit(pages, p.entry, p.unit, G, kH);
        const int64_t hq0 = (int64_t)unit.b * Hq + unit.h * G + unit.g0;
        const int each = (take + me.csize - 1) / me.csize, t0 = p.tile + min(me.crank * each, take);
        const int t1 = min(p.tile + min((me.crank + 1) * each, take), Line::tiles_with_rows(len));
        const int my_tiles = (t1 - t0 - warp + kWarps - 1) / kWarps;   // may be <= 0
        const int hp = pages.page_heads > 1 ? unit.h : 0;
        const T* kh = pages.k + hp * pages.head_stride;
        const T* vh = pages.v + hp * pages.head_stride;
        const int32_t* count = pages.count != nullptr ? pages.count + (int64_t)hp * pages.page_size : nullptr;
        Finder<false> finder = {pages.table_of(p.entry), pages.page_size, pages.page_bits, len, t0 + warp, my_tiles, {}, {}};
        finder.start(lane);
        const auto copy = [&](int stage_no, int j) {
            const uint32_t stage = ring + stage_no * stage_size;
            const int2 at = finder.get(j, lane);
            const bool page = pages.names_page(at.x);
            const int64_t mine = page ? at.x * pages.page_stride + (int64_t)at.y * pages.row_stride : -1;
            const unsigned rows_ok = __ballot_sync(kFull, page) & 0xffff;
            for (int r0 = 0; r0 < kTile; r0 += step) {
                const int r = r0 + v0;
                const int64_t o = __shfl_sync(kFull, mine, r);
                const uint32_t row = stage + r * pitch;
#pragma unroll
                for (int n = 0; n < kChunks; ++n) {
                    const int c = c0 + n * 32;
                    if (c >= chunks) continue;
                    const uint32_t to = row + ((c ^ (r & 7)) << 4);
                    cp_async16(to, o >= 0 ? (const void*)(kh + o + c * E) : q, o >= 0 ? 16 : 0);
                    cp_async16(to + kTile * pitch, o >= 0 ? (const void*)(vh + o + c * E) : q, o >= 0 ? 16 : 0);
                }
            }
            if (count != nullptr && lane < kTile) {
                const int64_t o = (int64_t)at.x * pages.page_heads * pages.page_size + at.y;
                cp_async4(stage + 2 * kTile * pitch + lane * 4, page ? (const void*)(count + o) : q, page ? 4 : 0);
            }
            if (lane == 0) asm volatile("st.shared.u32 [%0], %1;\n" ::"r"(stage + 2 * kTile * pitch + 64), "r"(rows_ok) : "memory");
            if (!page && (t0 + warp + j * kWarps) * kTile + (lane & 15) < len) set_status(status, SC_ERR_INVALID_ARG);
        };
#pragma unroll
        for (int s = 0; s < kStages; ++s) {
            if (s < my_tiles) copy(s, s);
            cp_async_commit();
        }
        for (int i = threadIdx.x; i < kH * d; i += kThreads) {
            const int g = i / d;
            sq[i] = g < unit.nh ? Elem<T>::load(q + hq0 * d + i) : 0.f;
        }
        __syncthreads();
        float m[kH], l[kH], acc[kH][kChunks][E];
#pragma unroll
        for (int g = 0; g < kH; ++g) {
            m[g] = -INFINITY; l[g] = 0.f;   // l: this lane's rows only
#pragma unroll
            for (int n = 0; n < kChunks; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[g][n][e] = 0.f;
        }
        int at_stage = 0;
        for (int i = 0; i < my_tiles; ++i) {
            cp_async_wait<kStages - 1>();
            __syncwarp();
            const unsigned char* st = ring_p + at_stage * stage_size;
            const int r = lane & 15;
            const bool ok = *reinterpret_cast<const unsigned*>(st + 2 * kTile * pitch + 64) >> r & 1;
            float4 s[kH];   // four sums a score: short chains of roundings
#pragma unroll
            for (int g = 0; g < kH; ++g) s[g] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
            for (int c = lane >> 4; c < chunks; c += 2) {
                float kv[E];
                unpack(*reinterpret_cast<const uint4*>(st + r * pitch + ((c ^ (r & 7)) << 4)), kv);
#pragma unroll
                for (int g = 0; g < kH; ++g)
#pragma unroll
                    for (int e = 0; e < E; e += 4) {
                        const float4 qv = *reinterpret_cast<const float4*>(sq + g * d + c * E + e);
                        const float2 a = umma::fma2(make_float2(qv.x, qv.y), make_float2(kv[e], kv[e + 1]), make_float2(s[g].x, s[g].y));
                        const float2 b = umma::fma2(make_float2(qv.z, qv.w), make_float2(kv[e + 2], kv[e + 3]), make_float2(s[g].z, s[g].w));
                        s[g] = make_float4(a.x, a.y, b.x, b.y);
                    }
            }
            float x[kH];
            // ln s, in base-2 units (a valid row has count >= 1)
            const float lc = count != nullptr ? log2f((float)max(reinterpret_cast<const int*>(st + 2 * kTile * pitch)[r], 1)) : 0.f;
            bool higher = false;
#pragma unroll
            for (int g = 0; g < kH; ++g) {
                x[g] = (s[g].x + s[g].y) + (s[g].z + s[g].w);
                x[g] += __shfl_xor_sync(kFull, x[g], 16);
                x[g] = ok ? fmaf(x[g], scale_log2, lc) : -INFINITY;
                higher |= x[g] > m[g] + kMaxSlack;
            }
            if (__any_sync(kFull, higher)) {
#pragma unroll
                for (int g = 0; g < kH; ++g) {
                    float mx = x[g];
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
                    const float mn = fmaxf(m[g], mx), f = mn == -INFINITY ? 1.f : exp2f(m[g] - mn);
                    l[g] *= f;
#pragma unroll
                    for (int n = 0; n < kChunks; ++n)
#pragma unroll
                        for (int e = 0; e < E; ++e) acc[g][n][e] *= f;
                    m[g] = mn;
                }
            }
#pragma unroll
            for (int g = 0; g < kH; ++g) {
                const float w = exp2f(x[g] - (m[g] == -INFINITY ? 0.f : m[g]));
                if (lane < 16) { l[g] += w; sp[warp][r][g] = w; }
            }
            __syncwarp();
#pragma unroll 4
            for (int r0 = 0; r0 < kTile; r0 += step) {
                const int vr = r0 + v0;
                float w[kH];
#pragma unroll
                for (int g = 0; g < kH; g += 4) {
                    const float4 t = *reinterpret_cast<const float4*>(&sp[warp][vr][g]);
                    w[g] = t.x; w[g + 1] = t.y; w[g + 2] = t.z; w[g + 3] = t.w;
                }
#pragma unroll
                for (int n = 0; n < kChunks; ++n) {
                    const int c = c0 + n * 32;
                    if (c >= chunks) continue;
                    float vv[E];
                    unpack(*reinterpret_cast<const uint4*>(st + (kTile + vr) * pitch + ((c ^ (vr & 7)) << 4)), vv);
#pragma unroll
                    for (int g = 0; g < kH; ++g)
#pragma unroll
                        for (int e = 0; e < E; e += 2) {
                            const float2 a = umma::fma2(make_float2(w[g], w[g]), make_float2(vv[e], vv[e + 1]), make_float2(acc[g][n][e], acc[g][n][e + 1]));
                            acc[g][n][e] = a.x; acc[g][n][e + 1] = a.y;
                        }
                }
            }
            __syncwarp();
            if (i + kStages < my_tiles) copy(at_stage, i + kStages);   // the stage just consumed takes the next tile
            cp_async_commit();
            at_stage = at_stage + 1 == kStages ? 0 : at_stage + 1;
        }
        cp_async_wait<0>();

        // ---- the warps of this block meet (fixed order) ----
#pragma unroll
        for (int g = 0; g < kH; ++g) {
            const float lw = warp_sum(l[g]);
            if (lw != lw) m[g] = fmaxf(m[g], 0.f);   // (no score was a number: not to be taken for a part without rows)
            if (lane == 0) { sh_m[warp][g] = m[g]; sh_l[warp][g] = lw; }
        }
        if (kH < kHeads && lane < kHeads - kH) { sh_m[warp][kH + lane] = -INFINITY; sh_l[warp][kH + lane] = 0.f; }
        __syncthreads();   // every warp is done with its ring; reuse it as [warp][kH][d] fp32
        float* slabs = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int g = 0; g < kH; ++g) {
            float bm = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) bm = fmaxf(bm, sh_m[w][g]);
            const float f = m[g] == -INFINITY ? 0.f : exp2f(m[g] - bm);
#pragma unroll
            for (int n = 0; n < kChunks; ++n)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float a = acc[g][n][e];
                    for (int o = width; o < 32; o <<= 1) a += __shfl_xor_sync(kFull, a, o);   // the lanes that share a chunk
                    const int c = c0 + n * 32;
                    if (v0 == 0 && c < chunks) slabs[(warp * kH + g) * d + c * E + e] = a * f;
                }
        }
        __syncthreads();
        const auto block_sum = [&](int e4) {   // four columns of a head
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(slabs + w * kH * d + e4 * 4);
                a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
            }
            return a;
        };
        const auto block_ml = [&](int g) {
            float bm = -INFINITY, bl = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) bm = fmaxf(bm, sh_m[w][g]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) bl += sh_m[w][g] == -INFINITY ? 0.f : sh_l[w][g] * exp2f(sh_m[w][g] - bm);
            return make_float2(bm, bl);
        };
        joiner.join(me, p, nt, take, unit.nh, d, out + hq0 * d, block_sum, block_ml);
        me.left -= take;
        if (me.left == 0) break;
        next_unit(line, p, nt);
        joiner.next(me);   // the ring, sq, sh_m and sh_l are written again
    }
    zero_empty(pages, line, Hq, G, kH, d, out);
    joiner.leave(me);
}

template <typename T, int kH, int kStages>
int bytes_of(int cluster, int d) { return kWarps * kStages * stage_bytes(pitch_of(d, sizeof(T))) + kH * d * 4 + (cluster > 1 ? 2 * recv_bytes(d, kH) : 0); }

template <typename T, int kH, int kStages, int kChunks>
cudaError_t start(const PagedDecodeArgs& a, cudaStream_t st) {
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    static std::once_flag once[64];   // per device
    static cudaError_t ready[64];
    const auto kernel = paged_decode_generic<T, kH, kStages, kChunks>;
    constexpr int kMost = kChunks * 32 * 16 / (int)sizeof(T) < kMaxD ? kChunks * 32 * 16 / (int)sizeof(T) : kMaxD;   // d
    std::call_once(once[dev & 63], [&] { ready[dev & 63] = opt_in(kernel, bytes_of<T, kH, kStages>(4, kMost), false); });
    if (ready[dev & 63] != cudaSuccess) return ready[dev & 63];
    Line line;
    line.lens = a.lens; line.entries = a.B * a.cache.table_heads; line.per_entry = a.Hkv / a.cache.table_heads * div_up(a.Hq / a.Hkv, kH);
    line.cap = a.cache.max_pages * a.cache.page_size;
    const Division part = divide(line, sms, [](int cluster, int d) {
        const int room = 228 * 1024 / (bytes_of<T, kH, kStages>(cluster, d) + 2560 + (kH > 4 ? 1024 : 0));
        return room < 1 ? 1 : room < blocks_by_registers(kH) ? room : blocks_by_registers(kH);
    }, a.d, false);
    const float scale = (a.scale == 0.f ? 1.f / sqrtf((float)a.d) : a.scale) * 1.4426950408889634f;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(line.parties * part.cluster);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes_of<T, kH, kStages>(part.cluster, a.d);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = part.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return own_error(cudaLaunchKernelEx(&cfg, kernel, pages_of<const T>(a.cache), (const T*)a.q, a.Hq, a.Hkv, a.d, line, part, scale, (T*)a.out,
                                        (int32_t*)a.ws, (float*)((char*)a.ws + kTicketBytes), a.status));
}

template <int kH>
cudaError_t start(const PagedDecodeArgs& a, cudaStream_t st) {
    typedef __nv_bfloat16 bf16;
    const int stages = stages_of(pitch_of(a.d, a.dt == SC_BF16 ? 2 : 4));
    if (a.dt == SC_BF16) return stages == 3 ? start<bf16, kH, 3, 1>(a, st) : stages == 2 ? start<bf16, kH, 2, 1>(a, st) : start<bf16, kH, 1, 1>(a, st);
    if (a.d > 128) return start<float, kH, 1, 2>(a, st);
    return stages == 3 ? start<float, kH, 3, 1>(a, st) : stages == 2 ? start<float, kH, 2, 1>(a, st) : start<float, kH, 1, 1>(a, st);
}

}  // namespace

}  // namespace pg

cudaError_t launch_paged_decode_generic(const PagedDecodeArgs& a, cudaStream_t st) {
    const cudaError_t e = a.Hq / a.Hkv <= 4 ? pg::start<4>(a, st) : pg::start<8>(a, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
