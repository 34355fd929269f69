// Tensor-core bf16 decode attention over a paged cache (Eq. 4; d = 64, 128 or 256; up to eight query heads at a time), sm_100a.
//
// The rows of all heads form one line of 16-row tiles (paged.cuh).  A party, a cluster of blocks (or one block), takes a stretch
// of it; its blocks share each segment's tiles out evenly and their warps take them in turn, each through a private ring of
// cp.async stages in shared memory (16-byte chunks, XOR-swizzled so that ldmatrix is conflict free).  Per tile:
//     S^T[16 keys x 8 heads]   = K_tile . q^T                (mma.m16n8k16, keys on M, heads on N)
//     x = S^T * scale*log2(e) + log2(count)
//     P^T = 2^(x - m)          (online softmax in fp32; the running maximum is common to the warp and raised only when a score
//                               overtakes it by a margin, so weights stay below 2^8)
//     O^T[d x 8 heads] += V_tile^T . P^T                     (P as a bf16 pair, leading part + remainder: sixteen bits of each weight)
// The sum of weights is taken over the same sixteen bits, so a weight's rounding moves the output towards or away from its own row only: some 2e-6
// of it, a thousandth of the rounding to bf16 that follows (an output that close to the middle between two bf16 values may go to the other).  A third bf16 of each weight
// would take a product more.
// Up to four query heads stand in the eight columns twice, the second time for the remainders.  Warps meet in shared memory, blocks of a
// cluster hand each other slices of their sums through distributed shared memory (decode_fold.cuh), parties that share a unit leave
// partial sums in global memory, slice by slice, and the last to arrive joins them.  Every order is fixed: results are bit-reproducible.
#include <mutex>

#include "paged_attn.cuh"

namespace sc {
namespace pg {

namespace {

typedef __nv_bfloat16 bf16;

constexpr float kMaxSlack = 8.f;          // log2 units a score may exceed the running maximum before it is raised

template <int D>
struct Shape {
    static constexpr int kStages = D == 64 ? 6 : 3;                  // about 96 KB on their way per block (192 for d = 256)
    static constexpr int kBlocksPerSm = D == 256 ? 1 : 2;
    static constexpr int kRowBytes = D * 2;
    static constexpr int kTileBytes = kTile * kRowBytes;             // of K or V
    static constexpr int kStageBytes = 2 * kTileBytes + 64;          // K, V, 16 counts
    static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
    static constexpr int kSmemBytes = kRingBytes + 2 * recv_bytes(D, kHeads);
    static_assert(kWarps * kHeads * D * 4 <= kRingBytes, "the warps' sums lie in the ring's place");
};
static_assert(kMaxBlocks * 4 <= (int)kTicketBytes, "a counter per party and slice");

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ float fast_log2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
// One head's rows as a warp copies them: tile after tile into stages.
template <int D, bool kWhole>
struct Rows {
    const bf16* k; const bf16* v;      // of the head inside the pages
    const int32_t* count;              // likewise, or NULL
    const void* nowhere;               // a valid address for copies of no bytes
    int64_t page_stride, row_stride;
    int64_t count_page;
    int num_pages, len;
    int32_t* status;

    // Where a tile lies, worked out before its stage is free (the lookup and the 64-bit products take as long as a product's step).
    struct Tile {
        int64_t first;      // kWhole: of the lane's first chunk, in elements; else of row lane & 15, or -1
        int64_t count;      // of the lane's count
        unsigned rows_ok;
    };
    __device__ __forceinline__ Tile locate(int tile, int2 at, int lane) const {
        constexpr int kChunks = D / 8;
        const bool page = (unsigned)at.x < (unsigned)num_pages;
        Tile t;
        if (kWhole) {
            const int rows = page ? min(kTile, len - tile * kTile) : 0;
            t.rows_ok = (1u << rows) - 1;
            t.first = at.x * page_stride + (int64_t)(at.y + lane / kChunks) * row_stride + lane % kChunks * 8;
        } else {
            t.rows_ok = __ballot_sync(kFull, page) & 0xffff;
            t.first = page ? at.x * page_stride + (int64_t)at.y * row_stride : -1;
        }
        t.count = at.x * count_page + at.y + (kWhole ? lane : 0);
        if (!page && tile * kTile + (kWhole ? 0 : lane & 15) < len) set_status(status, SC_ERR_INVALID_ARG);
        return t;
    }
    __device__ __forceinline__ void copy(uint32_t stage, const Tile& t, int lane) const {
        constexpr int kChunks = D / 8, kStep = 32 / kChunks, kN = kTile / kStep;   // lanes per row, rows per round, rounds
        using S = Shape<D>;
        const int c = lane % kChunks, r0 = lane / kChunks;
        const uint32_t dst = stage + r0 * S::kRowBytes;
        if (kWhole && t.rows_ok == 0xffff) {
            const bf16* ks = k + t.first;
            const bf16* vs = v + t.first;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const uint32_t to = dst + i * kStep * S::kRowBytes + ((c ^ ((i * kStep + r0) & 7)) << 4);
                cp_async16(to, ks, 16);
                cp_async16(to + S::kTileBytes, vs, 16);
                ks += kStep * row_stride; vs += kStep * row_stride;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const uint32_t to = dst + i * kStep * S::kRowBytes + ((c ^ ((i * kStep + r0) & 7)) << 4);
                const bool ok = t.rows_ok >> (i * kStep + r0) & 1;
                const int64_t o = kWhole ? t.first + (int64_t)i * kStep * row_stride : __shfl_sync(kFull, t.first, i * kStep + r0) + c * 8;
                cp_async16(to, ok ? (const void*)(k + o) : nowhere, ok ? 16 : 0);
                cp_async16(to + S::kTileBytes, ok ? (const void*)(v + o) : nowhere, ok ? 16 : 0);
            }
        }
        if (count != nullptr && lane < kTile) {
            const bool ok = t.rows_ok >> lane & 1;
            cp_async4(stage + 2 * S::kTileBytes + lane * 4, ok ? (const void*)(count + t.count) : nowhere, ok ? 4 : 0);
        }
    }
};

// kPair: up to four query heads (see above).
template <int D, bool kWhole, bool kPair>
__global__ void __launch_bounds__(kThreads, Shape<D>::kBlocksPerSm)
paged_decode_mma(const Pages<const bf16> pages, const bf16* __restrict__ q, int Hq, int Hkv, Line line, const Division how, float scale_log2,
                 bf16* __restrict__ out, int32_t* __restrict__ tickets, float* __restrict__ part, int32_t* status) {
    using S = Shape<D>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float sh_m[kWarps][kHeads], sh_l[kWarps][kHeads];
    __shared__ unsigned sh_rows[kWarps][8];    // which rows of a warp's tiles count, by turns
    __shared__ int sh_last;
    __shared__ __align__(8) unsigned long long sh_bar[2];   // what the cluster's blocks hand this one, segments by turns

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, tig = lane & 3;
    Party me;
    me.set_up(sh_bar);
    in_stream_order();
    const int G = Hq / Hkv;
    if (!me.plan(line, how, lane)) {
        zero_empty(pages, line, Hq, G, kHeads, D, out);
        me.step();
        return;
    }
    Joiner joiner = {sh_bar, smem + S::kRingBytes, &sh_last, tickets, part, status, kHeads, 0u, true};

    // per-lane ldmatrix row/chunk selectors
    const int lm_j = lane >> 3, lm_r = lane & 7;
    const int k_row = lm_r + ((lm_j & 1) << 3), k_csel = lm_j >> 1;    // K: matrices (r0-7,c), (r8-15,c), (r0-7,c+1), (r8-15,c+1)
    const int v_row = lm_r + ((lm_j >> 1) << 3), v_csel = lm_j & 1;    // V^T: (r0-7,c), (r0-7,c+1), (r8-15,c), (r8-15,c+1)
    const uint32_t ring = smem_u32(smem) + warp * (S::kStages * S::kStageBytes);

    // Up to four query heads: the warps' sums have a place of their own (the receiving places of a block that stands for itself), so the next
    // segment's first tiles are on their way while this one's warps meet (512 units of 24 tiles 29.2 us, 30.3 without).
    constexpr bool kApart = kPair && D <= 128;
    constexpr int kCols = kPair ? 4 : kHeads;            // columns of a warp's sums
    static_assert(!kApart || kWarps * kCols * D * 4 <= 2 * recv_bytes(D, kHeads), "");
    const bool apart = kApart && me.csize == 1;
    float* slabs = reinterpret_cast<float*>(apart ? smem + S::kRingBytes : smem);

    struct Segment {
        Place p;
        int nt, take, first, tiles, nh;   // the unit's tiles, the segment's; this warp's: first, first + kWarps, ...
        int64_t hq0;
        Rows<D, kWhole> rows;
        Finder<kWhole> finder;
    };
    const auto prepare = [&](const Place& p, unsigned left) {
        Segment s;
        const int len = line.len(p.entry);
        s.p = p;
        s.nt = line.tiles_of(len);
        s.take = (int)min((unsigned)(s.nt - p.tile), left);
        const Unit unit(pages, p.entry, p.unit, G, kHeads);
        s.nh = unit.nh;
        s.hq0 = (int64_t)unit.b * Hq + unit.h * G + unit.g0;
        const int each = (s.take + me.csize - 1) / me.csize, t0 = p.tile + min(me.crank * each, s.take);
        const int t1 = min(p.tile + min((me.crank + 1) * each, s.take), Line::tiles_with_rows(len));
        s.first = t0 + warp;
        s.tiles = (t1 - t0 - warp + kWarps - 1) / kWarps;   // may be <= 0
        const int hp = pages.page_heads > 1 ? unit.h : 0;
        s.rows.k = pages.k + hp * pages.head_stride; s.rows.v = pages.v + hp * pages.head_stride;
        s.rows.count = pages.count != nullptr ? pages.count + (int64_t)hp * pages.page_size : nullptr;
        s.rows.count_page = (int64_t)pages.page_heads * pages.page_size;
        s.rows.nowhere = q;
        s.rows.page_stride = pages.page_stride; s.rows.row_stride = pages.row_stride;
        s.rows.num_pages = pages.num_pages; s.rows.len = len; s.rows.status = status;
        s.finder = {pages.table_of(p.entry), pages.page_size, pages.page_bits, len, s.first, s.tiles, {}, {}};
        s.finder.start(lane);
        return s;
    };
    // the warp's j-th tile: found, and which of its rows count left where the products look (eight places: more than there are stages)
    const auto locate = [&](Segment& s, int j) __attribute__((always_inline)) {
        const auto tile = s.rows.locate(s.first + j * kWarps, s.finder.get(j, lane), lane);
        if (lane == 0) sh_rows[warp][j & 7] = tile.rows_ok;
        return tile;
    };
    static_assert(S::kStages < 8, "");
    const auto fill = [&](Segment& s) __attribute__((always_inline)) {   // the whole ring
#pragma unroll
        for (int i = 0; i < S::kStages; ++i) {
            if (i < s.tiles) s.rows.copy(ring + i * S::kStageBytes, locate(s, i), lane);
            cp_async_commit();
        }
    };

    Segment seg = prepare(me.begin(line, lane), me.left);
    fill(seg);
    for (;;) {
        const int my_tiles = seg.tiles, nh = seg.nh;
        const int64_t hq0 = seg.hq0;
        const bool last = me.left == (unsigned)seg.take;
        Segment then;
        if (apart && !last) {            // (its pages are looked up meanwhile)
            Place p = seg.p;
            next_unit(line, p, seg.nt);
            then = prepare(p, me.left - seg.take);
        }
        // q^T as the B operand of every k-step: b0 = q[head g][16ks + 2tig, +1], b1 = same + 8
        uint32_t qb[D / 16][2];
        {
            const int hd = kPair ? g & 3 : g;
            const bf16* qh = q + (hq0 + hd) * D + 2 * tig;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                qb[ks][0] = hd < nh ? *reinterpret_cast<const uint32_t*>(qh + ks * 16) : 0u;
                qb[ks][1] = hd < nh ? *reinterpret_cast<const uint32_t*>(qh + ks * 16 + 8) : 0u;
            }
        }
        float o[D / 16][4];
#pragma unroll
        for (int mt = 0; mt < D / 16; ++mt) { o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f; }
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;   // columns 2tig and 2tig+1

        int at_stage = 0;
        for (int i = 0; i < my_tiles; ++i) {
            typename Rows<D, kWhole>::Tile next = {};
            const bool more = i + S::kStages < my_tiles;
            if (more) next = locate(seg, i + S::kStages);
            cp_async_wait<S::kStages - 1>();   // tile i has landed, the next ones are on their way
            __syncwarp();
            const uint32_t st = ring + at_stage * S::kStageBytes;
            const unsigned char* st_p = smem + warp * (S::kStages * S::kStageBytes) + at_stage * S::kStageBytes;

            // S^T = K . q^T, four accumulator chains
            float s[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint32_t a[4];
                const int c = 2 * ks + k_csel;
                ldmatrix_x4(st + k_row * S::kRowBytes + ((c ^ (k_row & 7)) << 4), a);
                mma_bf16(s[ks & 3], a, qb[ks][0], qb[ks][1]);
            }
            const unsigned rows_ok = sh_rows[warp][i & 7];
            float lc_lo = 0.f, lc_hi = 0.f;
            if (seg.rows.count != nullptr) {
                const int* cs = reinterpret_cast<const int*>(st_p + 2 * S::kTileBytes);
                lc_lo = fast_log2((float)max(cs[g], 1));
                lc_hi = fast_log2((float)max(cs[g + 8], 1));
            }
            const bool ok_lo = rows_ok >> g & 1, ok_hi = rows_ok >> (g + 8) & 1;
            const float x0 = ok_lo ? fmaf((s[0][0] + s[1][0]) + (s[2][0] + s[3][0]), scale_log2, lc_lo) : -INFINITY;
            const float x1 = ok_lo ? fmaf((s[0][1] + s[1][1]) + (s[2][1] + s[3][1]), scale_log2, lc_lo) : -INFINITY;
            const float x2 = ok_hi ? fmaf((s[0][2] + s[1][2]) + (s[2][2] + s[3][2]), scale_log2, lc_hi) : -INFINITY;
            const float x3 = ok_hi ? fmaf((s[0][3] + s[1][3]) + (s[2][3] + s[3][3]), scale_log2, lc_hi) : -INFINITY;
            const float lx0 = fmaxf(x0, x2), lx1 = fmaxf(x1, x3);
            if (__any_sync(kFull, (lx0 > m0 + kMaxSlack) || (lx1 > m1 + kMaxSlack))) {
                float mx0 = lx0, mx1 = lx1;
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) {
                    mx0 = fmaxf(mx0, __shfl_xor_sync(kFull, mx0, off));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(kFull, mx1, off));
                }
                const float mn0 = fmaxf(m0, mx0), mn1 = fmaxf(m1, mx1);
                const float c0 = mn0 == -INFINITY ? 1.f : dm::fast_exp2(m0 - mn0), c1 = mn1 == -INFINITY ? 1.f : dm::fast_exp2(m1 - mn1);
                l0 *= c0; l1 *= c1;
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt) { o[mt][0] *= c0; o[mt][2] *= c0; o[mt][1] *= c1; o[mt][3] *= c1; }
                m0 = mn0; m1 = mn1;
            }
            const float e0 = m0 == -INFINITY ? 0.f : m0, e1 = m1 == -INFINITY ? 0.f : m1;   // (a tile whose page does not exist has no row)
            const float w0 = dm::fast_exp2(x0 - e0), w1 = dm::fast_exp2(x1 - e1);   // row g
            const float w2 = dm::fast_exp2(x2 - e0), w3 = dm::fast_exp2(x3 - e1);   // row g + 8
            const uint32_t p_lo = pack_bf16x2(w0, w1), p_hi = pack_bf16x2(w2, w3);
            const uint32_t r_lo = pack_bf16x2(w0 - bf16_lo(p_lo), w1 - bf16_hi(p_lo));
            const uint32_t r_hi = pack_bf16x2(w2 - bf16_lo(p_hi), w3 - bf16_hi(p_hi));
            l0 += (bf16_lo(p_lo) + bf16_lo(r_lo)) + (bf16_lo(p_hi) + bf16_lo(r_hi));
            l1 += (bf16_hi(p_lo) + bf16_hi(r_lo)) + (bf16_hi(p_hi) + bf16_hi(r_hi));
            const uint32_t pb0 = movmatrix_trans(kPair && tig >= 2 ? r_lo : p_lo), pb1 = movmatrix_trans(kPair && tig >= 2 ? r_hi : p_hi);
            const uint32_t rb0 = kPair ? 0u : movmatrix_trans(r_lo), rb1 = kPair ? 0u : movmatrix_trans(r_hi);

            // O^T += V^T . P^T
#pragma unroll
            for (int mt = 0; mt < D / 16; ++mt) {
                uint32_t a[4];
                const int c = 2 * mt + v_csel;
                ldmatrix_x4_trans(st + S::kTileBytes + v_row * S::kRowBytes + ((c ^ (v_row & 7)) << 4), a);
                mma_bf16(o[mt], a, pb0, pb1);
                if (!kPair) mma_bf16(o[mt], a, rb0, rb1);
            }
            __syncwarp();
            // the stage just consumed takes the next tile
            if (more) seg.rows.copy(st, next, lane);
            cp_async_commit();
            at_stage = at_stage + 1 == S::kStages ? 0 : at_stage + 1;
        }
        if (apart && !last) fill(then); else cp_async_wait<0>();

        // ---- the warps of this block meet (fixed order) ----
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {   // lane-local l covers rows g, g+8 of every tile
            l0 += __shfl_xor_sync(kFull, l0, off);
            l1 += __shfl_xor_sync(kFull, l1, off);
        }
        if (l0 != l0) m0 = fmaxf(m0, 0.f);   // (no score was a number: not to be taken for a part without rows)
        if (l1 != l1) m1 = fmaxf(m1, 0.f);
        if (g == 0) {
            sh_m[warp][2 * tig] = m0; sh_m[warp][2 * tig + 1] = m1;
            sh_l[warp][2 * tig] = l0; sh_l[warp][2 * tig + 1] = l1;
        }
        __syncthreads();   // every warp is done with its ring: its place, or another one, takes [warp][columns][D] fp32
        float bm0 = -INFINITY, bm1 = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { bm0 = fmaxf(bm0, sh_m[w][2 * tig]); bm1 = fmaxf(bm1, sh_m[w][2 * tig + 1]); }
        const float f0 = m0 == -INFINITY ? 0.f : dm::fast_exp2(m0 - bm0), f1 = m1 == -INFINITY ? 0.f : dm::fast_exp2(m1 - bm1);
        float* slab = slabs + warp * (kCols * D);
#pragma unroll
        for (int mt = 0; mt < D / 16; ++mt) {
            const int d0 = mt * 16 + g;
            float v[4] = {o[mt][0] * f0, o[mt][1] * f1, o[mt][2] * f0, o[mt][3] * f1};
            if (kPair) {   // the remainders' part (their columns' maxima are the same)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += __shfl_xor_sync(kFull, v[i], 2);
                if (tig >= 2) continue;
            }
            slab[(2 * tig) * D + d0] = v[0];
            slab[(2 * tig + 1) * D + d0] = v[1];
            slab[(2 * tig) * D + d0 + 8] = v[2];
            slab[(2 * tig + 1) * D + d0 + 8] = v[3];
        }
        __syncthreads();
        const auto block_sum = [&](int e4) {   // four columns of a head: e4 = head * D / 4 + column / 4
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(slabs + w * (kCols * D) + e4 * 4);
                acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
            }
            return acc;
        };
        const auto block_ml = [&](int hd) {
            float bm = -INFINITY, bl = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) bm = fmaxf(bm, sh_m[w][hd]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) bl += sh_m[w][hd] == -INFINITY ? 0.f : sh_l[w][hd] * dm::fast_exp2(sh_m[w][hd] - bm);
            return make_float2(bm, bl);
        };
        joiner.join(me, seg.p, seg.nt, seg.take, nh, D, out + hq0 * D, block_sum, block_ml);
        if (last) break;
        me.left -= seg.take;
        joiner.next(me);   // the sums' place, sh_m and sh_l are written again, and the ring where it is that place
        if (apart) {
            seg = then;
        } else {
            Place p = seg.p;
            next_unit(line, p, seg.nt);
            seg = prepare(p, me.left);
            fill(seg);
        }
    }
    zero_empty(pages, line, Hq, G, kHeads, D, out);
    joiner.leave(me);
}

template <int D, bool kWhole, bool kPair>
cudaError_t start(const PagedDecodeArgs& a, Line line, int dev, int sms, cudaStream_t st) {
    static std::once_flag once[64];   // per device
    static cudaError_t ready[64];
    std::call_once(once[dev & 63], [dev] {
        ready[dev & 63] = opt_in(paged_decode_mma<D, kWhole, kPair>, Shape<D>::kSmemBytes, false);
    });
    if (ready[dev & 63] != cudaSuccess) return ready[dev & 63];
    const Division part = divide(line, sms, [](int, int) { return Shape<D>::kBlocksPerSm; }, D, Shape<D>::kBlocksPerSm > 1);
    const int c = part.cluster;
    const float scale = (a.scale == 0.f ? 1.f / sqrtf((float)a.d) : a.scale) * 1.4426950408889634f;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(line.parties * c);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Shape<D>::kSmemBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = c; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return own_error(cudaLaunchKernelEx(&cfg, paged_decode_mma<D, kWhole, kPair>, pages_of<const bf16>(a.cache), (const bf16*)a.q, a.Hq, a.Hkv, line, part,
                                        scale, (bf16*)a.out, (int32_t*)a.ws, (float*)((char*)a.ws + kTicketBytes), a.status));
}

template <int D>
cudaError_t start(const PagedDecodeArgs& a, const Line& line, int dev, int sms, cudaStream_t st) {
    const bool whole = a.cache.page_size % kTile == 0, pair = a.Hq / a.Hkv <= 4;
    return whole ? (pair ? start<D, true, true>(a, line, dev, sms, st) : start<D, true, false>(a, line, dev, sms, st))
                 : (pair ? start<D, false, true>(a, line, dev, sms, st) : start<D, false, false>(a, line, dev, sms, st));
}

}  // namespace

Division divide(Line& line, int sms, int (*blocks_of)(int cluster, int d), int d, bool one_per_sm) {
    const int64_t units = (int64_t)line.entries * line.per_entry;
    // Up to 64 units: clusters of four, as many as find room at once (7/8 of the block slots: 64 of 4 x 74), and of those a multiple of the units
    // where that costs little, so that stretches of equal lengths end where units end.  us, against single blocks two per SM: 8 units of 8 K rows 13.2
    // and 18.7, of 32 K 29.5 and 35.1, of 128 K 91 and 99; 4 units of 128 K with seven query heads 52 and 76; 32 units of 15 K 49.6 and 53.5.  Clusters
    // of eight: 1 K rows 7.8 and 9.8 (of four), but 8 K 15.7 and 13.2, because the next launch's clusters find room only when this one is gone.
    // From 17 units on each block stands for itself where the units are short: 32 units of 3 K rows 18.3 (clusters 21), of 25 K 81 and 81.
    // More units: single blocks, two per SM (128 units of 150 rows 12.8, in clusters of two 17.1); where units are long one per SM, which reads
    // fewer streams at a time (128 units of 6 K rows 71.8 and 73.9, of 12 K 124 and 128, of 16 K 166 and 175; but 512 of 1.5 K 73.0 and 69.7, 2048 of
    // 400 rows 111 and 78; 128 units of 3 K and 512 of 3 K the same).
    // Tables of no more than 2.5 K rows, up to 16 units: clusters of eight, one per unit (8 units of 2 K rows 8.1, two clusters a unit 8.9, clusters of four
    // 8.9; 16 units of 2.3 K rows 9.4, 12.3 with two; 8 of 0.5 K 5.9, of four 7.0).  This goes by the tables' width, since lengths are known on the device
    // only: the same rows in tables for 128 K rows take clusters of four (8 units of 2 K 9.1, 16 of 2.3 K 9.9, 8 of 0.5 K 7.0).
    line.spare = 0;
    const bool small = units <= 16 && line.tiles_of(line.cap) <= 5 * 8 * kWarps;
    const int c = small ? 8 : units <= 64 ? 4 : 1;
    int blocks = sms * blocks_of(c, d);
    if (blocks > kMaxBlocks) blocks = kMaxBlocks;
    // Many units per block: what a unit costs besides its rows counts as a round more, so that a block with many short ones has fewer rows (256 sequences
    // of 20 to 200 rows 48.7 -> 39 us, 512 of 10 to 100 63 -> 58, 80 of 150 to 500 30.2 -> 28.3; but 64 of 20 to 200, 512 units on 296 blocks, 15.1 -> 15.9).
    line.spare = c == 1 && units > 2 * blocks ? kWarps : 0;
    unsigned short_below = 0;
    line.parties = blocks;
    if (c > 1) {
        line.parties = blocks * 7 / 8 / c;
        int64_t most = (units * line.tiles_of(line.cap) + c * kWarps * kLeast - 1) / (c * kWarps * kLeast);   // what full tables could occupy
        if (most < units || small) most = units;
        if (most < line.parties) line.parties = (int)most;
        if (units <= line.parties && 8 * (line.parties % units) <= line.parties) line.parties -= (int)(line.parties % units);
        short_below = units <= 16 ? 0 : (unsigned)units * 512;
    }
    return {c, short_below, c == 1 && one_per_sm && units < 0x1000000 ? (unsigned)units * kLongUnit : 0xffffffffu, sms};
}

}  // namespace pg

bool paged_decode_mma_supported(const PagedDecodeArgs& a) { return a.dt == SC_BF16 && (a.d == 64 || a.d == 128 || a.d == 256); }

size_t paged_decode_ws_bytes() { return pg::kTicketBytes + sizeof(float) * 2 * pg::kMaxBlocks * pg::part_floats(pg::kMaxD); }

cudaError_t launch_paged_decode_mma(const PagedDecodeArgs& a, cudaStream_t st) {
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    pg::Line line;
    line.lens = a.lens; line.entries = a.B * a.cache.table_heads;
    line.per_entry = a.Hkv / a.cache.table_heads * div_up(a.Hq / a.Hkv, pg::kHeads);
    line.cap = a.cache.max_pages * a.cache.page_size;
    const cudaError_t e = a.d == 64 ? pg::start<64>(a, line, dev, sms, st) : a.d == 128 ? pg::start<128>(a, line, dev, sms, st) : pg::start<256>(a, line, dev, sms, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
