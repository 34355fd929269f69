// sc_paged_decode_attn for any type and head size (d a multiple of 8 up to 256): one pass over the rows on CUDA cores.
//
// One block takes a stretch of the launch's line of tiles (paged.cuh), for up to four query heads of a KV head at a time.  Its warps
// take 32-row tiles of a segment in turn: a lane finds the page of one row; eight lanes per row form the scores, one
// lane per row takes part in the online softmax in fp32, and for the weighted sum a lane owns four columns of every row.
// Serves SC_F32 and head sizes that the tensor-core kernel does not take, and cross-checks it.
#include "paged.cuh"

namespace sc {
namespace pg {

namespace {

constexpr int kTile = 32;
constexpr int kHeads = 4;       // query heads per block
constexpr int kMaxD = 256;
constexpr int kWarps = 4;
constexpr int kPartiesPerSm = 3;
constexpr int kMaxParties = 160 * kPartiesPerSm;
constexpr int kLeast = 4;       // tiles a stretch has at least: one per warp

static_assert(kMaxParties * 4 <= (int)kTicketBytes, "a counter per party");

// NC: the most 32-column pieces a row has (4 or 8).
template <typename T, int NC>
__global__ void __launch_bounds__(kWarps * 32)
paged_decode_generic(const Pages<T> pages, const T* __restrict__ q, int Hq, int Hkv, int d, const Line line, float scale_log2, T* __restrict__ out,
                     int32_t* __restrict__ tickets, float* __restrict__ part, int32_t* status) {
    constexpr int kPer = NC / 4;
    __shared__ __align__(16) float sq[kHeads][kMaxD];
    __shared__ __align__(16) float4 sp[kWarps][kTile];              // scores, then weights, of a tile: [row][head]
    __shared__ __align__(16) float so[kWarps][kHeads][kMaxD];       // the warps' sums
    __shared__ float sm[kWarps][kHeads], sl[kWarps][kHeads];
    __shared__ int sh_last;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, sub = lane & 7, rsub = lane >> 3;
    in_stream_order();
    const int G = Hq / Hkv, groups = (G + kHeads - 1) / kHeads, ps = pages.page_size;
    const auto head_of = [&](int entry, int unit, int& b, int& h, int& g0) {
        b = entry / pages.table_heads;
        h = pages.table_heads > 1 ? entry - b * pages.table_heads : unit / groups;
        g0 = unit % groups * kHeads;
    };
    // heads without rows
    for (int e = blockIdx.x; e < line.entries; e += gridDim.x) {
        if (line.len(e) > 0) continue;
        for (int i = threadIdx.x; i < line.per_entry * kHeads * d; i += kWarps * 32) {
            int b, h, g0;
            const int unit = i / (kHeads * d), g = i / d % kHeads;
            head_of(e, unit, b, h, g0);
            if (g0 + g < G) Elem<T>::store(out + ((int64_t)b * Hq + h * G + g0 + g) * d + i % d, 0.f);
        }
    }
    const unsigned total = total_of(line, lane), stretch = max((total + line.parties - 1) / line.parties, (unsigned)kLeast), from = min((uint64_t)blockIdx.x * stretch, (uint64_t)total);
    if (from >= total) return;
    unsigned left = min(stretch, total - from);
    for (Place p = place_of(line, from, lane);;) {
        const int len = line.len(p.entry), nt = line.tiles(p.entry);
        const int take = (int)min((unsigned)(nt - p.tile), left), t_end = p.tile + take;
        int b, h, g0;
        head_of(p.entry, p.unit, b, h, g0);
        const int nh = min(kHeads, G - g0), hq0 = b * Hq + h * G + g0;
        const int32_t* table = pages.table_of(p.entry);
        const int hp = pages.page_heads > 1 ? h : 0;
        const T* kh = pages.k + hp * pages.head_stride;
        const T* vh = pages.v + hp * pages.head_stride;
        for (int i = threadIdx.x; i < kHeads * kMaxD; i += kWarps * 32) {
            const int g = i / kMaxD, c = i % kMaxD;
            sq[g][c] = g < nh && c < d ? Elem<T>::load(q + (int64_t)(hq0 + g) * d + c) * scale_log2 : 0.f;
        }
        __syncthreads();
        float m[kHeads], l[kHeads], acc[kHeads][kPer][4];
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
            m[g] = -INFINITY; l[g] = 0.f;   // l: this lane's rows only
#pragma unroll
            for (int u = 0; u < kPer; ++u) acc[g][u][0] = acc[g][u][1] = acc[g][u][2] = acc[g][u][3] = 0.f;
        }
        for (int t = p.tile + w; t < t_end; t += kWarps) {
            const int row = t * kTile + lane;
            int64_t at = -1;   // where this lane's row lies
            float lc = 0.f;    // ln s, in base-2 units
            if (row < len) {
                const int slot = row / ps, id = table[slot];
                if (pages.names_page(id)) {
                    at = id * pages.page_stride + (int64_t)(row - slot * ps) * pages.row_stride;
                    if (pages.count != nullptr) lc = log2f((float)max(pages.count[((int64_t)id * pages.page_heads + hp) * ps + (row - slot * ps)], 1));
                } else {
                    set_status(status, SC_ERR_INVALID_ARG);
                }
            }
            const unsigned rows_ok = __ballot_sync(kFull, at >= 0);
#pragma unroll (16 / NC)
            for (int it = 0; it < 8; ++it) {   // four rows at a time
                const int r = it * 4 + rsub;
                const int64_t ra = __shfl_sync(kFull, at, r);
                float4 kv[NC];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int col = (c * 8 + sub) * 4;
                    kv[c] = ra >= 0 && col < d ? load4(kh + ra + col) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                float s[kHeads];
#pragma unroll
                for (int g = 0; g < kHeads; ++g) {
                    s[g] = 0.f;
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const float4 qv = *reinterpret_cast<const float4*>(&sq[g][(c * 8 + sub) * 4]);
                        s[g] = fmaf(qv.x, kv[c].x, fmaf(qv.y, kv[c].y, fmaf(qv.z, kv[c].z, fmaf(qv.w, kv[c].w, s[g]))));
                    }
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1)
#pragma unroll
                    for (int g = 0; g < kHeads; ++g) s[g] += __shfl_xor_sync(kFull, s[g], o);
                if (sub == 0) sp[w][r] = make_float4(s[0], s[1], s[2], s[3]);
            }
            __syncwarp();
            {
                const float4 xs = sp[w][lane];
                const float x[kHeads] = {xs.x, xs.y, xs.z, xs.w};
                float pw[kHeads];
#pragma unroll
                for (int g = 0; g < kHeads; ++g) {
                    const float xg = rows_ok >> lane & 1 ? x[g] + lc : -INFINITY;
                    const float mn = fmaxf(m[g], warp_max(xg)), ref = mn == -INFINITY ? 0.f : mn;   // (no row so far)
                    const float corr = exp2f(m[g] - ref);
                    pw[g] = exp2f(xg - ref);
                    l[g] = l[g] * corr + pw[g];
#pragma unroll
                    for (int u = 0; u < kPer; ++u) { acc[g][u][0] *= corr; acc[g][u][1] *= corr; acc[g][u][2] *= corr; acc[g][u][3] *= corr; }
                    m[g] = mn;
                }
                __syncwarp();
                sp[w][lane] = make_float4(pw[0], pw[1], pw[2], pw[3]);
            }
            __syncwarp();
#pragma unroll
            for (int r0 = 0; r0 < kTile; r0 += 16) {   // sixteen rows requested together
                if ((rows_ok >> r0 & 0xffff) == 0) continue;
#pragma unroll
                for (int u = 0; u < kPer; ++u) {
                    const int col = (u * 32 + lane) * 4;
                    float4 vv[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int64_t ra = __shfl_sync(kFull, at, r0 + j);
                        vv[j] = ra >= 0 && col < d ? load4(vh + ra + col) : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float4 pv = sp[w][r0 + j];
                        const float pgv[kHeads] = {pv.x, pv.y, pv.z, pv.w};
#pragma unroll
                        for (int g = 0; g < kHeads; ++g) {
                            acc[g][u][0] = fmaf(pgv[g], vv[j].x, acc[g][u][0]); acc[g][u][1] = fmaf(pgv[g], vv[j].y, acc[g][u][1]);
                            acc[g][u][2] = fmaf(pgv[g], vv[j].z, acc[g][u][2]); acc[g][u][3] = fmaf(pgv[g], vv[j].w, acc[g][u][3]);
                        }
                    }
                }
            }
            __syncwarp();   // the next tile's scores overwrite the weights
        }
        // the warps' (m, l, O), in order
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
            const float lw = warp_sum(l[g]);
            if (lane == 0) { sm[w][g] = m[g]; sl[w][g] = lw; }
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int col = (u * 32 + lane) * 4;
                *reinterpret_cast<float4*>(&so[w][g][col]) = make_float4(acc[g][u][0], acc[g][u][1], acc[g][u][2], acc[g][u][3]);
            }
        }
        __syncthreads();
        const bool whole = take == nt;
        const int part_stride = kHeads * (d + 2);
        float* mine = part + (size_t)(2 * blockIdx.x + (p.at > from)) * part_stride;   // [head][d columns, m, l]
        for (int i = threadIdx.x; i < nh * d; i += kWarps * 32) {
            const int g = i / d, c = i - g * d;
            float mm = -INFINITY;
#pragma unroll
            for (int j = 0; j < kWarps; ++j) mm = fmaxf(mm, sm[j][g]);
            float ls = 0.f, o = 0.f;
#pragma unroll
            for (int j = 0; j < kWarps; ++j) {
                const float f = sm[j][g] == -INFINITY ? 0.f : exp2f(sm[j][g] - mm);   // 0: a warp without rows
                ls += f * sl[j][g];
                o = fmaf(f, so[j][g][c], o);
            }
            if (whole) {
                Elem<T>::store(out + (int64_t)(hq0 + g) * d + c, ls != 0.f ? o / ls : 0.f);
            } else {
                mine[g * (d + 2) + c] = o;
                if (c == 0) { mine[g * (d + 2) + d] = mm; mine[g * (d + 2) + d + 1] = ls; }
            }
        }
        if (!whole) {
            const unsigned first = p.at / stretch, last = (p.at + nt - 1) / stretch;
            int32_t* ticket = tickets + first;   // (a party begins one shared unit at most)
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                int t;
                asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;\n" : "=r"(t) : "l"(ticket) : "memory");
                sh_last = t == (int)(last - first);
                if (sh_last) *ticket = 0;   // ready for the next call
            }
            __syncthreads();
            if (sh_last) {
                for (int i = threadIdx.x; i < nh * d; i += kWarps * 32) {
                    const int g = i / d, c = i - g * d;
                    float mm = -INFINITY, ls = 0.f, o = 0.f;
                    for (unsigned j = first; j <= last; ++j) {
                        const float* from_j = part + (size_t)(2 * j + (p.at > j * stretch)) * part_stride + g * (d + 2);
                        const float mj = __ldcg(from_j + d), lj = __ldcg(from_j + d + 1), oj = __ldcg(from_j + c);
                        const float mn = fmaxf(mm, mj), ref = mn == -INFINITY ? 0.f : mn;
                        const float c0 = exp2f(mm - ref), c1 = exp2f(mj - ref);
                        ls = ls * c0 + lj * c1;
                        o = o * c0 + oj * c1;
                        mm = mn;
                    }
                    Elem<T>::store(out + (int64_t)(hq0 + g) * d + c, ls != 0.f ? o / ls : 0.f);
                }
            }
        }
        left -= take;
        if (left == 0) return;
        next_unit(line, p, nt);
        __syncthreads();   // sq, so, sm, sl are written again
    }
}

template <typename T>
cudaError_t run(const PagedDecodeArgs& a, cudaStream_t st) {
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const Pages<T> pages = pages_of<T>(a.cache);
    const int groups = div_up(a.Hq / a.Hkv, kHeads);
    Line line;
    line.lens = a.lens; line.entries = a.B * a.cache.table_heads; line.per_entry = a.Hkv / a.cache.table_heads * groups;
    line.cap = pages.cap(); line.tile = kTile;
    line.parties = sms * kPartiesPerSm < kMaxParties ? sms * kPartiesPerSm : kMaxParties;
    const float scale = (a.scale == 0.f ? 1.f / sqrtf((float)a.d) : a.scale) * 1.4426950408889634f;
    return launch_in_order(a.d <= 128 ? paged_decode_generic<T, 4> : paged_decode_generic<T, 8>, dim3(line.parties), kWarps * 32, 0, st, pages,
                           (const T*)a.q, a.Hq, a.Hkv, a.d, line, scale, (T*)a.out, (int32_t*)a.ws, (float*)((char*)a.ws + kTicketBytes), a.status);
}

}  // namespace

}  // namespace pg

size_t paged_decode_generic_ws_bytes(int32_t d) {
    return pg::kTicketBytes + sizeof(float) * 2 * pg::kMaxParties * pg::kHeads * ((size_t)d + 2);
}

cudaError_t launch_paged_decode_generic(const PagedDecodeArgs& a, cudaStream_t st) {
    const cudaError_t e = a.dt == SC_BF16 ? pg::run<__nv_bfloat16>(a, st) : pg::run<float>(a, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
