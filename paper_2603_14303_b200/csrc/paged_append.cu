// sc_paged_append: new rows of a ragged batch go into the pages of their sequences, keys and queries rotated on the way.
//
// One block serves one piece of one sequence: the new rows that fall into one page (without bounds: into 64 rows of it), for some of the
// heads (keys, values and queries counted in one row).  So a page's bounds belong to one block per head, whose warps hold whole heads: smallest and
// largest key are taken in registers over the piece's rows, as stored and two at a time in bf16, and meet in a few shuffles; no atomics.  The host knows T and B only, from which
// follow the most pieces there can be; which piece is a block's own it finds by counting all sequences' pieces.  (Places for two pieces more than
// n / page_size per sequence, found without counting, were half empty where every sequence has one token: 256 of them 9.3 us, counted 5.9.  Every block
// counts the sequences before its own, 256 at a time: 2000 single tokens 51 us, 4096 (four heads) 80.)
// Sines and cosines of a piece's rows are taken once per block, 16 rows at a time, and shared by its heads.
#include <limits.h>

#include <type_traits>

#include "paged.cuh"

namespace sc {
namespace pg {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSub = 16;          // rows whose sines and cosines are held at a time
constexpr int kMaxHalf = 128;     // most pairs of a row
constexpr int kGroupHeads = 32;   // most heads (keys, values, queries) per block
constexpr int kCutRows = 64;

// The smaller and the larger; not a number where one is not (a page with such a key must not lose it).
__device__ __forceinline__ float min_nan(float a, float b) { float y; asm("min.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ uint32_t min_nan2(uint32_t a, uint32_t b) { uint32_t y; asm("min.NaN.bf16x2 %0, %1, %2;\n" : "=r"(y) : "r"(a), "r"(b)); return y; }
__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) { uint32_t y; asm("max.NaN.bf16x2 %0, %1, %2;\n" : "=r"(y) : "r"(a), "r"(b)); return y; }

template <typename T, int E> struct Vec;
template <> struct Vec<__nv_bfloat16, 8> {
    uint4 w;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(a[i] << 16); x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        uint32_t a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            a[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
        w = make_uint4(a[0], a[1], a[2], a[3]);
    }
    __device__ __forceinline__ void fill(float x) { const float v[8] = {x, x, x, x, x, x, x, x}; set(v); }
    __device__ __forceinline__ void lower(const Vec& o) { w = make_uint4(min_nan2(w.x, o.w.x), min_nan2(w.y, o.w.y), min_nan2(w.z, o.w.z), min_nan2(w.w, o.w.w)); }
    __device__ __forceinline__ void raise(const Vec& o) { w = make_uint4(max_nan2(w.x, o.w.x), max_nan2(w.y, o.w.y), max_nan2(w.z, o.w.z), max_nan2(w.w, o.w.w)); }
    __device__ __forceinline__ Vec from(int o) const {
        Vec v;
        v.w = make_uint4(__shfl_xor_sync(kFull, w.x, o), __shfl_xor_sync(kFull, w.y, o), __shfl_xor_sync(kFull, w.z, o), __shfl_xor_sync(kFull, w.w, o));
        return v;
    }
};
template <> struct Vec<float, 4> {
    float4 w;
    __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = w; }
    __device__ __forceinline__ void get(float (&x)[4]) const { x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w; }
    __device__ __forceinline__ void set(const float (&x)[4]) { w = make_float4(x[0], x[1], x[2], x[3]); }
    __device__ __forceinline__ void fill(float x) { w = make_float4(x, x, x, x); }
    __device__ __forceinline__ void lower(const Vec& o) { w = make_float4(min_nan(w.x, o.w.x), min_nan(w.y, o.w.y), min_nan(w.z, o.w.z), min_nan(w.w, o.w.w)); }
    __device__ __forceinline__ void raise(const Vec& o) { w = make_float4(max_nan(w.x, o.w.x), max_nan(w.y, o.w.y), max_nan(w.z, o.w.z), max_nan(w.w, o.w.w)); }
    __device__ __forceinline__ Vec from(int o) const {
        Vec v;
        v.w = make_float4(__shfl_xor_sync(kFull, w.x, o), __shfl_xor_sync(kFull, w.y, o), __shfl_xor_sync(kFull, w.z, o), __shfl_xor_sync(kFull, w.w, o));
        return v;
    }
};
template <typename T> struct Vec<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T* p) { w = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = w; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = Elem<T>::load(&w); }
    __device__ __forceinline__ void set(const float (&x)[1]) { Elem<T>::store(&w, x[0]); }
    __device__ __forceinline__ void fill(float x) { Elem<T>::store(&w, x); }
    __device__ __forceinline__ void lower(const Vec& o) { fill(min_nan(Elem<T>::load(&w), Elem<T>::load(&o.w))); }
    __device__ __forceinline__ void raise(const Vec& o) { fill(max_nan(Elem<T>::load(&w), Elem<T>::load(&o.w))); }
    __device__ __forceinline__ Vec from(int o) const { Vec v; v.fill(__shfl_xor_sync(kFull, Elem<T>::load(&w), o)); return v; }
};

// Angles are taken in turns as 64-bit fixed-point fractions, whose wrap-around is the whole turns': the step of a pair, freq / 2 pi, once per block
// and pair in two doubles (1 / 2 pi = kTurn + kTurnRest to 107 bits), off by 2^-62.6 of a turn, then one integer product per position, off by 2^-31.6
// of a turn at the farthest position (2^31), 2^-45 at 128 K.  It is cut to 2^-32 of a turn and rounded to 24 bits, at most 2^-26 of a turn, for
// sincospif.  (In doubles per position and pair it was a quarter of all instructions of a long prompt.)
constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;
__device__ __forceinline__ uint64_t turn_step(float freq) {
    const double f = freq, hi = f * kTurn, lo = fma(f, kTurn, -hi) + f * kTurnRest;
    const double part = hi - rint(hi);                      // exact, in [-1/2, 1/2]
    return (uint64_t)(int64_t)rint(part * 0x1p62) * 4 + (uint64_t)(int64_t)rint(lo * 0x1p64);   // (2^62: 2^63 is no int64)
}
__device__ __forceinline__ float2 turn(int position, uint64_t step) {
    const int32_t t = (int32_t)(((uint64_t)(int64_t)position * step) >> 32);   // in 2^-32 turns
    float s, c;
    sincospif((float)t * 0x1p-31f, &s, &c);
    return make_float2(c, s);
}

struct News { int first, n, have; bool fits; };   // a sequence's new rows: the first token, how many (-1: they break the rules), rows before, room
struct Dims { int B, Hq, Hkv, T, d, group, cut, cuts; };   // cut: most rows of a piece, page_size or 64; cuts: pieces of a page

// E: elements of a vector.  kUnits: units of a row (see below) where they fill a power of two of lanes and all columns are rotated, or none; 0: any.
// kBounds: the pages' bounds are kept, in some 110 registers, so two blocks per SM; without them three fit (32 K tokens 161 -> 135 us).  With bounds a
// third block costs spills (four prompts of 64-row pages 154 -> 190 us), as it does in the kernel for any units (11.0 -> 13.4 us).
template <typename T, int E, bool kPairs, int kUnits, bool kBounds>
__global__ void __launch_bounds__(kThreads, kBounds || kUnits == 0 ? 2 : 3) append_paged(const Pages<T> pages, const sc_paged_rows rows, const Dims dims, int32_t* status) {
    // Cosines and sines of a row, in the order in which lanes take them: lane u the pairs u * E .. u * E + E - 1, four at a time, so that
    // each four of neighbouring lanes lie side by side (as a plain list of pairs, read with 16-way bank conflicts, 35 K tokens x 48 heads took 265 us).
    __shared__ __align__(16) float sh_cos[kSub * kMaxHalf], sh_sin[kSub * kMaxHalf];
    __shared__ uint64_t sh_step[kMaxHalf];
    __shared__ News sh_news;
    __shared__ int sh_seq, sh_piece, sh_sums[kWarps], sh_tops[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = pages.page_size, B = dims.B, Hkv = dims.Hkv, d = dims.d;
    if (tid == 0) sh_seq = -1;
    in_stream_order();
    __syncthreads();
    const int rot = rows.inv_freq != nullptr ? rows.rot_dim : 0, half = rot / 2;
    for (int i = tid; i < half; i += kThreads) sh_step[i] = turn_step(rows.inv_freq[i]);
    const auto news_of = [&](int b, bool& falls) {
        const int o0 = rows.seq_off[b], o1 = rows.seq_off[b + 1], have = rows.cache_len[b];
        falls = o1 < o0;
        const int n = rows.seq_len != nullptr ? rows.seq_len[b] : o1 - o0;
        const bool valid = o0 >= 0 && o1 >= o0 && o1 <= dims.T && n >= 0 && n <= o1 - o0 && have >= 0;
        return News{o0, valid ? n : -1, have, valid && (n == 0 || (int64_t)have + n <= pages.cap())};   // (no rows: they fit)
    };
    const auto tell = [&](int b, const News& w) {
        if (!w.fits) set_status(status, w.n >= 0 ? SC_ERR_CAPACITY : SC_ERR_INVALID_ARG);
        if (rows.len_out != nullptr) rows.len_out[b] = w.fits ? w.have + w.n : w.have;
    };
    // pieces of `cut` rows of every page, numbered along a sequence's rows
    const unsigned cuts = dims.cuts;              // of a page
    const auto piece_of = [&](unsigned row) {     // (a length near 2^31 and rows that do not fit: below 2^32)
        const unsigned page = row / (unsigned)ps;
        return cuts == 1 ? page : page * cuts + (row - page * ps) / (unsigned)dims.cut;
    };
    // Sequences are counted in rounds of kThreads; those of the rounds x, x + gridDim.x, ... are told by block x.  Where offsets fall (then all rounds are
    // gone through again, carefully) a sequence whose tokens start before an offset in front of its own is at fault too: ranges that lie apart have
    // no more pieces than there are blocks, and no token is two sequences'.
    const unsigned n_rounds = ((unsigned)B + kThreads - 1) / kThreads;
    const auto count = [&](auto careful) {           // whether it has to be done carefully
        unsigned tells = blockIdx.y == 0 ? blockIdx.x : n_rounds;
        int before = 0, top = INT_MIN;               // pieces of the sequences so far; their largest offset
        for (unsigned round = 0; round < n_rounds && (before <= (int)blockIdx.x || tells < n_rounds); ++round) {
            const int b = (int)(round * kThreads + tid);
            const bool is = (unsigned)b < (unsigned)B;   // (past 2^31 - 1 in the last round of the largest batches)
            News w = {0, 0, 0, false};
            bool falls = false;
            if (is) w = news_of(b, falls);
            if constexpr (careful) {
                int most = warp_scan_max(is ? w.first : INT_MIN, lane);
                if (lane == 31) sh_tops[warp] = most;
                __syncthreads();
                most = max(most, top);
                for (int i = 0; i < kWarps; ++i) {
                    if (i < warp) most = max(most, sh_tops[i]);
                    top = max(top, sh_tops[i]);
                }
                if (is && w.first < most) { w.n = -1; w.fits = false; }
            }
            const int pieces = w.n > 0 ? (int)(piece_of((unsigned)w.have + w.n - 1) - piece_of(w.have)) + 1 : 0;
            const int upto = warp_scan_add(pieces, lane);
            const bool again = !careful && __any_sync(kFull, falls);
            if (lane == 31) sh_sums[warp] = again ? -1 : upto;
            __syncthreads();
            int first = before + upto - pieces, signs = 0;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                const int sum = sh_sums[i];
                first += i < warp ? sum : 0;
                before += sum;
                signs |= sum;
            }
            if (!careful && signs < 0) return true;
            if ((unsigned)((int)blockIdx.x - first) < (unsigned)pieces) { sh_seq = b; sh_piece = (int)blockIdx.x - first; sh_news = w; }
            __syncthreads();
            if (round == tells) {
                if (is) tell(b, w);
                tells += gridDim.x;
            }
        }
        return false;
    };
    if (count(std::false_type())) {
        __syncthreads();                             // (sh_sums is written again)
        count(std::true_type());
    }
    const int b = sh_seq;
    if (b < 0) return;
    const int o0 = sh_news.first, have = sh_news.have, n = sh_news.n;
    const bool fits = sh_news.fits;
    // the piece: rows [r0, r1) of the sequence, of the page whose first row is p0 (64 bits: a length near 2^31 with rows that do not fit)
    const unsigned piece = piece_of(have) + sh_piece, slot = cuts == 1 ? piece : piece / cuts;
    const int64_t p0 = (int64_t)slot * ps, c0 = p0 + (int64_t)(piece - slot * cuts) * dims.cut;
    const int64_t r0 = c0 > have ? c0 : have, r1 = min(min(c0 + dims.cut, p0 + ps), (int64_t)have + n);
    if (r0 >= r1) return;
    const int nr = (int)(r1 - r0), in_page = (int)(r0 - p0), tok0 = o0 + (int)(r0 - have);
    int id = -1;
    if (fits) {
        id = pages.table_of(b)[slot];
        if (!pages.names_page(id)) {
            id = -1;
            if (blockIdx.y == 0 && tid == 0) set_status(status, SC_ERR_INVALID_ARG);
        }
    }
    const int heads = 2 * Hkv + (rows.q != nullptr ? dims.Hq : 0);
    int h_lo = blockIdx.y * dims.group;
    const int h_hi = min(h_lo + dims.group, heads);
    if (id < 0) h_lo = max(h_lo, 2 * Hkv);   // queries only
    if (h_lo >= h_hi) return;

    // A row is d / E vectors, taken two at a time: a unit is the two that rotate into each other (or two neighbours).
    const int n_vec = kUnits ? 2 * kUnits : d / E, rot_units = kUnits ? (kPairs || half == 0 ? 0 : kUnits) : kPairs ? 0 : half / E;
    const int units = kUnits ? kUnits : rot_units + (n_vec - 2 * rot_units + 1) / 2;
    int unit_lanes = kUnits ? kUnits : 1;
    while (!kUnits && unit_lanes < units && unit_lanes < 32) unit_lanes *= 2;
    const int slots = 32 / unit_lanes;      // rows, or rows of several heads, a warp holds at once
    int row_slots = 1;
    while (row_slots < nr && row_slots < slots) row_slots *= 2;
    const int head_slots = slots / row_slots;
    const int lu = lane % unit_lanes, lr = lane / unit_lanes % row_slots, lh = lane / (unit_lanes * row_slots);
    constexpr int kFour = E < 4 ? 1 : 4;
    const int turned_units = (half + E - 1) / E, cs_row = turned_units * E;
    const auto place_of_pair = [&](int c) { return (c % E / kFour * turned_units + c / E) * kFour + c % kFour; };
    const int64_t page_at = (int64_t)id * pages.page_stride;
    const bool bounds = kBounds && id >= 0;

    for (int s0 = 0; s0 < nr; s0 += kSub) {
        const int ns = min(kSub, nr - s0);
        if (s0 > 0) __syncthreads();   // everybody is done with the rows before
        for (int i = tid; i < ns * half; i += kThreads) {
            const int r = i / half, c = i - r * half;
            const int pos = rows.positions != nullptr ? rows.positions[tok0 + s0 + r] : (int)(r0 + s0 + r);
            const float2 t = turn(pos, sh_step[c]);
            sh_cos[r * cs_row + place_of_pair(c)] = t.x;
            sh_sin[r * cs_row + place_of_pair(c)] = t.y;
        }
        if (pages.count != nullptr && blockIdx.y == 0 && id >= 0)
            for (int i = tid; i < ns * Hkv; i += kThreads) {
                const int r = i / Hkv, h = i - r * Hkv;
                pages.count[((int64_t)id * pages.page_heads + h) * ps + in_page + s0 + r] =
                    rows.count != nullptr ? rows.count[(int64_t)(tok0 + s0 + r) * Hkv + h] : 1;
            }
        __syncthreads();
        for (int hb = h_lo + warp * head_slots; hb < h_hi; hb += kWarps * head_slots) {
            const int x = hb + lh;
            const bool active = x < h_hi, is_k = x < Hkv, is_v = !is_k && x < 2 * Hkv;
            const T* src; T* dst;
            int64_t src_row, dst_row;
            if (is_k || is_v) {
                const int h = is_k ? x : x - Hkv;
                src = static_cast<const T*>(is_k ? rows.k : rows.v) + (int64_t)(tok0 + s0) * rows.kv_token + h * rows.kv_head;
                dst = (is_k ? pages.k : pages.v) + page_at + h * pages.head_stride + (int64_t)(in_page + s0) * pages.row_stride;
                src_row = rows.kv_token; dst_row = pages.row_stride;
            } else {
                const int h = x - 2 * Hkv;
                src = static_cast<const T*>(rows.q) + (int64_t)(tok0 + s0) * rows.q_token + h * rows.q_head;
                dst = static_cast<T*>(rows.q_out) + (int64_t)(tok0 + s0) * rows.qo_token + h * rows.qo_head;
                src_row = rows.q_token; dst_row = rows.qo_token;
            }
            for (int u0 = 0; u0 < units; u0 += unit_lanes) {
                const int u = u0 + lu;
                const bool turned = !is_v && (kUnits ? half > 0 : kPairs ? 2 * u * E < rot : u < rot_units);
                const int va = u < rot_units ? u : 2 * rot_units + 2 * (u - rot_units), vb = u < rot_units ? u + rot_units : va + 1;
                const bool has_a = active && (kUnits || u < units), has_b = kUnits ? has_a : has_a && vb < n_vec;
                Vec<T, E> lo_a, hi_a, lo_b, hi_b;
                if (kBounds) { lo_a.fill(INFINITY); lo_b.fill(INFINITY); hi_a.fill(-INFINITY); hi_b.fill(-INFINITY); }
                for (int rb = lr; rb < ns; rb += 4 * row_slots) {   // four rows requested together
                    Vec<T, E> a[4], c[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = rb + j * row_slots;
                        const T* at = src + r * src_row;
                        if (r < ns && has_a) a[j].load(at + va * E);
                        if (r < ns && has_b) c[j].load(at + vb * E);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = rb + j * row_slots;
                        if (r >= ns || !has_a) continue;
                        if (turned) {
                            float xa[E], xb[E];
                            a[j].get(xa);
                            if (has_b) c[j].get(xb);
                            float cosv[E], sinv[E];
#pragma unroll
                            for (int f = 0; f < E / kFour; ++f) {
                                const int at = r * cs_row + (f * turned_units + u) * kFour;
                                if constexpr (kFour == 4) {
                                    const float4 x4 = *reinterpret_cast<const float4*>(sh_cos + at), y4 = *reinterpret_cast<const float4*>(sh_sin + at);
                                    cosv[4 * f] = x4.x; cosv[4 * f + 1] = x4.y; cosv[4 * f + 2] = x4.z; cosv[4 * f + 3] = x4.w;
                                    sinv[4 * f] = y4.x; sinv[4 * f + 1] = y4.y; sinv[4 * f + 2] = y4.z; sinv[4 * f + 3] = y4.w;
                                } else {
                                    cosv[f] = sh_cos[at]; sinv[f] = sh_sin[at];
                                }
                            }
                            if constexpr (kPairs) {   // (columns 2 u E on: pairs u E on)
#pragma unroll
                                for (int e = 0; e < E; ++e) {
                                    if (!kUnits && u * E + e >= half) break;
                                    float& x1 = e < E / 2 ? xa[2 * e] : xb[2 * e - E];
                                    float& x2 = e < E / 2 ? xa[2 * e + 1] : xb[2 * e - E + 1];
                                    const float y1 = x1 * cosv[e] - x2 * sinv[e], y2 = x2 * cosv[e] + x1 * sinv[e];
                                    x1 = y1; x2 = y2;
                                }
                            } else {
#pragma unroll
                                for (int e = 0; e < E; ++e) {
                                    const float y1 = xa[e] * cosv[e] - xb[e] * sinv[e], y2 = xb[e] * cosv[e] + xa[e] * sinv[e];
                                    xa[e] = y1; xb[e] = y2;
                                }
                            }
                            a[j].set(xa);
                            if (has_b) c[j].set(xb);
                        }
                        T* to = dst + r * dst_row;
                        a[j].store(to + va * E);
                        if (has_b) c[j].store(to + vb * E);
                        if (bounds && is_k) {   // of what is stored
                            lo_a.lower(a[j]); hi_a.raise(a[j]);
                            if (has_b) { lo_b.lower(c[j]); hi_b.raise(c[j]); }
                        }
                    }
                }
                if (!bounds || hb >= Hkv) continue;   // (the same for the whole warp)
                for (int o = unit_lanes; o < unit_lanes * row_slots; o *= 2) {
                    lo_a.lower(lo_a.from(o)); hi_a.raise(hi_a.from(o));
                    lo_b.lower(lo_b.from(o)); hi_b.raise(hi_b.from(o));
                }
                if (is_k && has_a && lr == 0) {
                    // a page whose first row is new starts afresh, another one's bounds are widened (the same thread comes back here with the next
                    // rows of a longer piece)
                    T* mn = pages.k_min + ((int64_t)id * pages.page_heads + x) * d;
                    T* mx = pages.k_max + ((int64_t)id * pages.page_heads + x) * d;
                    if (in_page + s0 > 0) {
                        Vec<T, E> old[4];
                        old[0].load(mn + va * E); old[1].load(mx + va * E);
                        if (has_b) { old[2].load(mn + vb * E); old[3].load(mx + vb * E); }
                        lo_a.lower(old[0]); hi_a.raise(old[1]);
                        if (has_b) { lo_b.lower(old[2]); hi_b.raise(old[3]); }
                    }
                    lo_a.store(mn + va * E); hi_a.store(mx + va * E);
                    if (has_b) { lo_b.store(mn + vb * E); hi_b.store(mx + vb * E); }
                }
            }
        }
    }
}

template <typename T, int E, bool kBounds>
auto kernel_for(bool pairs, int rot, int units) {
    // Two halves that are not whole vectors are rotated element by element.
    if (!pairs && (rot / 2) % E != 0) return append_paged<T, 1, false, 0, kBounds>;
    switch (units) {
        case 4: return pairs ? append_paged<T, E, true, 4, kBounds> : append_paged<T, E, false, 4, kBounds>;
        case 8: return pairs ? append_paged<T, E, true, 8, kBounds> : append_paged<T, E, false, 8, kBounds>;
        case 16: return pairs ? append_paged<T, E, true, 16, kBounds> : append_paged<T, E, false, 16, kBounds>;
        default: return pairs ? append_paged<T, E, true, 0, kBounds> : append_paged<T, E, false, 0, kBounds>;
    }
}

template <typename T, int E>
cudaError_t run(const PagedAppendArgs& a, cudaStream_t st) {
    const int heads = 2 * a.Hkv + (a.rows.q != nullptr ? a.Hq : 0);
    // heads per block: 32, or down to 8 where that leaves SMs idle
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    // A page's bounds belong to one block; without them long pages are shared out.  n rows touch n / page_size + 2 pages at most, n / cut + 2 + 1 per
    // page's end pieces of them, and no more than n.
    const int cut = a.cache.k_min != nullptr || a.cache.page_size < kCutRows ? a.cache.page_size : kCutRows;
    int64_t blocks = a.T / cut + 2ll * a.B + (cut < a.cache.page_size ? a.T / a.cache.page_size + 2ll * a.B : 0);
    if (blocks > a.T) blocks = a.T > 0 ? a.T : 1;
    const int64_t pieces = blocks < a.T / cut + a.B ? blocks : a.T / cut + a.B;   // about
    int64_t groups = div_up(heads, kGroupHeads);
    if (groups * pieces < 2 * sms) groups = 2 * sms / pieces < div_up(heads, 8) ? 2 * sms / pieces : div_up(heads, 8);
    const Dims dims = {a.B, a.Hq, a.Hkv, a.T, a.d, div_up(heads, groups), cut, div_up(a.cache.page_size, cut)};
    if (blocks > 0x7fffffff || groups > 65535) return cudaErrorInvalidConfiguration;
    const Pages<T> pages = pages_of<T>(a.cache);
    const dim3 grid((unsigned)blocks, (unsigned)groups);
    const bool pairs = (a.flags & SC_FLAG_ROPE_PAIRS) != 0;
    const int rot = a.rows.inv_freq != nullptr ? a.rows.rot_dim : 0, units = a.d % (2 * E) == 0 && (rot == 0 || rot == a.d) ? a.d / (2 * E) : 0;
    const auto kernel = a.cache.k_min != nullptr ? kernel_for<T, E, true>(pairs, rot, units) : kernel_for<T, E, false>(pairs, rot, units);
    return launch_in_order(kernel, grid, kThreads, 0, st, pages, a.rows, dims, a.status);
}

}  // namespace

}  // namespace pg

cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st) {
    const cudaError_t e = a.dt == SC_BF16 ? pg::run<__nv_bfloat16, 8>(a, st) : pg::run<float, 4>(a, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
