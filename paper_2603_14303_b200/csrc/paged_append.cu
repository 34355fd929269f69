// sc_paged_append: new rows of a ragged batch go into the pages of their sequences, keys and queries rotated on the way.
//
// One block serves one piece of one sequence: the new rows that fall into one page, for some of the heads (keys, values and
// queries counted in one row).  So a page's bounds belong to one block per head, whose warps hold whole heads: smallest and
// largest key are taken in registers over the piece's rows and meet in a few shuffles; no atomics.  The host knows T and B only:
// block x serves the sequence b with f(b) <= x < f(b + 1), f(b) = seq_off[b] / page_size + 2 b, and its piece x - f(b); n rows
// touch at most n / page_size + 2 pages, so every piece has a block, and every block finds its sequence with one look at the
// offsets.  Sines and cosines of a piece's rows are taken once per block, 16 rows at a time, and shared by its heads.
#include "paged.cuh"

namespace sc {
namespace pg {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSub = 16;          // rows whose sines and cosines are held at a time
constexpr int kMaxHalf = 128;     // most pairs of a row
constexpr int kGroupHeads = 32;   // most heads (keys, values, queries) per block

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
};
template <> struct Vec<float, 4> {
    float4 w;
    __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = w; }
    __device__ __forceinline__ void get(float (&x)[4]) const { x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w; }
    __device__ __forceinline__ void set(const float (&x)[4]) { w = make_float4(x[0], x[1], x[2], x[3]); }
};
template <typename T> struct Vec<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T* p) { w = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = w; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = Elem<T>::load(&w); }
    __device__ __forceinline__ void set(const float (&x)[1]) { Elem<T>::store(&w, x[0]); }
};

// The smaller and the larger; not a number where one is not (a page with such a key must not lose it).
__device__ __forceinline__ float min_nan(float a, float b) { float y; asm("min.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(a), "f"(b)); return y; }

// cos and sin of position * freq.  The product of an int32 and a float is exact in 64 bits; in turns (times 1 / 2 pi) its whole part is dropped
// there too, and what is left, at most half a turn, is exact enough in 32 bits whatever the position was.
__device__ __forceinline__ float2 turn(int position, float freq) {
    double t = (double)position * (double)freq * 0.15915494309189533577;
    t -= rint(t);
    float s, c;
    sincospif((float)(2.0 * t), &s, &c);
    return make_float2(c, s);
}

struct Dims { int B, Hq, Hkv, T, d, group; };

template <typename T, int E, bool kPairs>
__global__ void __launch_bounds__(kThreads) append_paged(const Pages<T> pages, const sc_paged_rows rows, const Dims dims, int32_t* status) {
    __shared__ float2 sh_cs[kSub * kMaxHalf];
    __shared__ int sh_seq;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = pages.page_size, B = dims.B, Hkv = dims.Hkv, d = dims.d;
    if (tid == 0) sh_seq = -1;
    in_stream_order();
    __syncthreads();
    for (int b = tid; b < B; b += kThreads) {
        const int o0 = rows.seq_off[b], o1 = rows.seq_off[b + 1];
        if (o0 < 0 || o1 < o0 || o1 > dims.T) {
            if (blockIdx.x == 0 && blockIdx.y == 0) set_status(status, SC_ERR_INVALID_ARG);
            continue;
        }
        const int64_t f0 = o0 / ps + 2ll * b, f1 = o1 / ps + 2ll * (b + 1);
        if (f0 <= blockIdx.x && blockIdx.x < f1) sh_seq = b;   // (offsets that do not fall: one sequence at most)
    }
    __syncthreads();
    const int b = sh_seq;
    if (b < 0) return;
    const int o0 = rows.seq_off[b], range = rows.seq_off[b + 1] - o0;
    const int piece = (int)(blockIdx.x - (o0 / ps + 2ll * b));
    const int n = rows.seq_len != nullptr ? rows.seq_len[b] : range;
    const int have = rows.cache_len[b];
    if (n < 0 || n > range || have < 0) {
        if (piece == 0 && blockIdx.y == 0 && tid == 0) {
            set_status(status, SC_ERR_INVALID_ARG);
            if (rows.len_out != nullptr) rows.len_out[b] = have;
        }
        return;
    }
    const bool fits = (int64_t)have + n <= pages.cap();
    if (piece == 0 && blockIdx.y == 0 && tid == 0) {
        if (!fits) set_status(status, SC_ERR_CAPACITY);
        if (rows.len_out != nullptr) rows.len_out[b] = fits ? have + n : have;
    }
    // the piece: rows [r0, r1) of the sequence (64 bits: a length near 2^31 with rows that do not fit)
    const int64_t slot = have / ps + (int64_t)piece, p0 = slot * ps;
    const int64_t r0 = p0 > have ? p0 : have, r1 = min(p0 + ps, (int64_t)have + n);
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
    const int rot = rows.inv_freq != nullptr ? rows.rot_dim : 0, half = rot / 2;
    const int heads = 2 * Hkv + (rows.q != nullptr ? dims.Hq : 0);
    int h_lo = blockIdx.y * dims.group;
    const int h_hi = min(h_lo + dims.group, heads);
    if (id < 0) h_lo = max(h_lo, 2 * Hkv);   // queries only
    if (h_lo >= h_hi) return;

    // A row is d / E vectors, taken two at a time: a unit is the two that rotate into each other (or two neighbours).
    const int n_vec = d / E, rot_units = kPairs ? 0 : half / E;
    const int units = rot_units + (n_vec - 2 * rot_units + 1) / 2;
    int unit_lanes = 1;
    while (unit_lanes < units && unit_lanes < 32) unit_lanes *= 2;
    const int slots = 32 / unit_lanes;      // rows, or rows of several heads, a warp holds at once
    int row_slots = 1;
    while (row_slots < nr && row_slots < slots) row_slots *= 2;
    const int head_slots = slots / row_slots;
    const int lu = lane % unit_lanes, lr = lane / unit_lanes % row_slots, lh = lane / (unit_lanes * row_slots);
    const int64_t page_at = (int64_t)id * pages.page_stride;
    const bool bounds = pages.k_min != nullptr && id >= 0;

    for (int s0 = 0; s0 < nr; s0 += kSub) {
        const int ns = min(kSub, nr - s0);
        if (s0 > 0) __syncthreads();   // everybody is done with the rows before
        for (int i = tid; i < ns * half; i += kThreads) {
            const int r = i / half, c = i - r * half;
            const int pos = rows.positions != nullptr ? rows.positions[tok0 + s0 + r] : (int)(r0 + s0 + r);
            sh_cs[i] = turn(pos, rows.inv_freq[c]);
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
                const bool turned = !is_v && (kPairs ? 2 * u * E < rot : u < rot_units);
                const int va = u < rot_units ? u : 2 * rot_units + 2 * (u - rot_units), vb = u < rot_units ? u + rot_units : va + 1;
                const bool has_a = active && u < units, has_b = has_a && vb < n_vec;
                float lo_a[E], hi_a[E], lo_b[E], hi_b[E];
#pragma unroll
                for (int e = 0; e < E; ++e) { lo_a[e] = lo_b[e] = INFINITY; hi_a[e] = hi_b[e] = -INFINITY; }
                for (int rb = lr; rb < ns; rb += 4 * row_slots) {   // four rows requested together
                    Vec<T, E> a[4], c[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = rb + j * row_slots;
                        if (r < ns && has_a) a[j].load(src + r * src_row + va * E);
                        if (r < ns && has_b) c[j].load(src + r * src_row + vb * E);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = rb + j * row_slots;
                        if (r >= ns || !has_a) continue;
                        if (turned) {
                            float xa[E], xb[E];
                            a[j].get(xa);
                            if (has_b) c[j].get(xb);
                            const float2* cs = sh_cs + r * half;
                            if constexpr (kPairs) {
#pragma unroll
                                for (int e = 0; e < E; e += 2) {
                                    const int pa = (va * E + e) / 2, pb = (vb * E + e) / 2;
                                    if (pa < half) {
                                        const float2 t = cs[pa];
                                        const float y1 = xa[e] * t.x - xa[e + 1] * t.y, y2 = xa[e + 1] * t.x + xa[e] * t.y;
                                        xa[e] = y1; xa[e + 1] = y2;
                                    }
                                    if (has_b && pb < half) {
                                        const float2 t = cs[pb];
                                        const float y1 = xb[e] * t.x - xb[e + 1] * t.y, y2 = xb[e + 1] * t.x + xb[e] * t.y;
                                        xb[e] = y1; xb[e + 1] = y2;
                                    }
                                }
                            } else {
#pragma unroll
                                for (int e = 0; e < E; ++e) {
                                    const float2 t = cs[u * E + e];
                                    const float y1 = xa[e] * t.x - xb[e] * t.y, y2 = xb[e] * t.x + xa[e] * t.y;
                                    xa[e] = y1; xb[e] = y2;
                                }
                            }
                            a[j].set(xa);
                            if (has_b) c[j].set(xb);
                        }
                        a[j].store(dst + r * dst_row + va * E);
                        if (has_b) c[j].store(dst + r * dst_row + vb * E);
                        if (bounds && is_k) {   // of what is stored
                            float xa[E], xb[E];
                            a[j].get(xa);
#pragma unroll
                            for (int e = 0; e < E; ++e) { lo_a[e] = min_nan(lo_a[e], xa[e]); hi_a[e] = max_nan(hi_a[e], xa[e]); }
                            if (has_b) {
                                c[j].get(xb);
#pragma unroll
                                for (int e = 0; e < E; ++e) { lo_b[e] = min_nan(lo_b[e], xb[e]); hi_b[e] = max_nan(hi_b[e], xb[e]); }
                            }
                        }
                    }
                }
                if (!bounds || hb >= Hkv) continue;   // (the same for the whole warp)
                for (int o = unit_lanes; o < unit_lanes * row_slots; o *= 2) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        lo_a[e] = min_nan(lo_a[e], __shfl_xor_sync(kFull, lo_a[e], o)); hi_a[e] = max_nan(hi_a[e], __shfl_xor_sync(kFull, hi_a[e], o));
                        lo_b[e] = min_nan(lo_b[e], __shfl_xor_sync(kFull, lo_b[e], o)); hi_b[e] = max_nan(hi_b[e], __shfl_xor_sync(kFull, hi_b[e], o));
                    }
                }
                if (is_k && has_a && lr == 0) {
                    // a page whose first row is new starts afresh; the same thread comes back here with the next rows of a longer piece
                    const bool widen = in_page + s0 > 0;
                    T* mn = pages.k_min + ((int64_t)id * pages.page_heads + x) * d;
                    T* mx = pages.k_max + ((int64_t)id * pages.page_heads + x) * d;
                    const auto put = [&](T* at, float (&v)[E], bool smaller) {
                        Vec<T, E> w;
                        if (widen) {
                            float old[E];
                            w.load(at);
                            w.get(old);
#pragma unroll
                            for (int e = 0; e < E; ++e) v[e] = smaller ? min_nan(v[e], old[e]) : max_nan(v[e], old[e]);
                        }
                        w.set(v);
                        w.store(at);
                    };
                    put(mn + va * E, lo_a, true);
                    put(mx + va * E, hi_a, false);
                    if (has_b) { put(mn + vb * E, lo_b, true); put(mx + vb * E, hi_b, false); }
                }
            }
        }
    }
}

template <typename T, int E>
cudaError_t run(const PagedAppendArgs& a, cudaStream_t st) {
    const int heads = 2 * a.Hkv + (a.rows.q != nullptr ? a.Hq : 0);
    const int groups = div_up(heads, kGroupHeads);
    const Dims dims = {a.B, a.Hq, a.Hkv, a.T, a.d, div_up(heads, groups)};
    const int64_t blocks = a.T / a.cache.page_size + 2ll * a.B;
    if (blocks > 0x7fffffff || groups > 65535) return cudaErrorInvalidConfiguration;
    const Pages<T> pages = pages_of<T>(a.cache);
    const dim3 grid((unsigned)blocks, groups);
    const bool pairs = (a.flags & SC_FLAG_ROPE_PAIRS) != 0;
    // Two halves that are not whole vectors are rotated element by element.
    if (!pairs && a.rows.inv_freq != nullptr && (a.rows.rot_dim / 2) % E != 0)
        return launch_in_order(append_paged<T, 1, false>, grid, kThreads, 0, st, pages, a.rows, dims, a.status);
    return launch_in_order(pairs ? append_paged<T, E, true> : append_paged<T, E, false>, grid, kThreads, 0, st, pages, a.rows, dims, a.status);
}

}  // namespace

}  // namespace pg

cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st) {
    const cudaError_t e = a.dt == SC_BF16 ? pg::run<__nv_bfloat16, 8>(a, st) : pg::run<float, 4>(a, st);
    if (e == cudaSuccess) note_launches(1);
    return e;
}

}  // namespace sc
