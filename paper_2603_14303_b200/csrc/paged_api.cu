// C-ABI entry points of the paged cache: argument validation and dispatch.  See include/semanticache.h.
#include <math.h>

#include <algorithm>

#include "paged.cuh"

using namespace sc;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
size_t esize(sc_dtype dt) { return dt == SC_BF16 ? 2 : 4; }
bool stride16(int64_t s, sc_dtype dt) { return s >= 0 && (s * esize(dt)) % 16 == 0; }

sc_status check_shape(sc_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t d) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || (Hq % Hkv) != 0) return SC_ERR_INVALID_ARG;
    if (dt != SC_BF16 && dt != SC_F32) return SC_ERR_UNSUPPORTED;
    if (d < 8 || d > 256 || (d % 8) != 0) return SC_ERR_UNSUPPORTED;
    if ((int64_t)B * Hq > 0x7fffffff) return SC_ERR_UNSUPPORTED;
    return SC_OK;
}

// The tables and the pool's sizes.
sc_status check_tables(const sc_paged_cache* c, int32_t Hkv) {
    if (c == nullptr || c->num_pages < 0 || c->page_size < 1 || c->max_pages < 0) return SC_ERR_INVALID_ARG;
    if ((int64_t)c->max_pages * c->page_size > 0x7fffffff) return SC_ERR_INVALID_ARG;
    if (c->page_heads != Hkv && c->page_heads != 1) return SC_ERR_INVALID_ARG;
    if (c->table_heads != Hkv && c->table_heads != 1) return SC_ERR_INVALID_ARG;
    if (c->page_heads != Hkv && c->table_heads != Hkv) return SC_ERR_INVALID_ARG;   // pages of one head need tables per head
    if (c->max_pages > 0 && (c->table == nullptr || c->table_stride < c->max_pages)) return SC_ERR_INVALID_ARG;
    return SC_OK;
}

// Where the rows lie.
sc_status check_pool(const sc_paged_cache* c, sc_dtype dt, int32_t d) {
    if (c->num_pages > 0 && (c->k == nullptr || c->v == nullptr)) return SC_ERR_INVALID_ARG;
    if (!aligned16(c->k) || !aligned16(c->v)) return SC_ERR_INVALID_ARG;
    if (!stride16(c->page_stride, dt) || !stride16(c->head_stride, dt) || !stride16(c->row_stride, dt)) return SC_ERR_INVALID_ARG;
    if (c->row_stride < d) return SC_ERR_INVALID_ARG;
    return SC_OK;
}

// Whether rows of d elements, one for every combination of the axes' indexes, lie apart: in order of their strides each axis of more than one entry
// steps over what the axes before it cover, as the axes of any permuted view do, with gaps or without.
struct Axis { int64_t n, stride; };
bool apart(int64_t d, Axis a, Axis b, Axis c = {1, 0}) {
    Axis axes[3] = {a, b, c};
    if (a.n == 0 || b.n == 0 || c.n == 0) return true;
    std::sort(axes, axes + 3, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
    __int128 covered = d;
    for (const Axis& x : axes) {
        if (x.n == 1) continue;
        if (x.stride < covered) return false;
        covered += (__int128)(x.n - 1) * x.stride;
    }
    return true;
}

}  // namespace

extern "C" {

sc_status sc_paged_append(const sc_paged_cache* cache, const sc_paged_rows* rows, sc_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t T,
                          int32_t d, uint32_t flags, int32_t* status, void* stream) {
    sc_status s = check_shape(dt, B, Hq, Hkv, d);
    if (s == SC_OK) s = check_tables(cache, Hkv);
    if (s == SC_OK) s = check_pool(cache, dt, d);
    if (s != SC_OK) return s;
    if (rows == nullptr || T < 0 || (flags & ~SC_FLAG_ROPE_PAIRS)) return SC_ERR_INVALID_ARG;
    if (cache->page_heads != Hkv || cache->table_heads != 1) return SC_ERR_INVALID_ARG;
    if (rows->rot_dim < 0 || rows->rot_dim > d || (rows->rot_dim & 1) != 0) return SC_ERR_INVALID_ARG;
    if ((rows->q == nullptr) != (rows->q_out == nullptr)) return SC_ERR_INVALID_ARG;
    if (rows->count != nullptr && cache->count == nullptr) return SC_ERR_INVALID_ARG;
    if ((cache->k_min == nullptr) != (cache->k_max == nullptr)) return SC_ERR_INVALID_ARG;
    if (!aligned16(cache->k_min) || !aligned16(cache->k_max)) return SC_ERR_INVALID_ARG;
    if (!apart(d, {cache->num_pages, cache->page_stride}, {cache->page_heads, cache->head_stride}, {cache->page_size, cache->row_stride})) return SC_ERR_INVALID_ARG;
    if (rows->q_out != nullptr && !apart(d, {T, rows->qo_token}, {Hq, rows->qo_head})) return SC_ERR_INVALID_ARG;
    if (B == 0) return SC_OK;
    if (rows->seq_off == nullptr || rows->cache_len == nullptr || rows->cache_len == rows->len_out) return SC_ERR_INVALID_ARG;
    if (T > 0 && (rows->k == nullptr || rows->v == nullptr)) return SC_ERR_INVALID_ARG;
    if (!aligned16(rows->k) || !aligned16(rows->v) || !aligned16(rows->q) || !aligned16(rows->q_out)) return SC_ERR_INVALID_ARG;
    if (!stride16(rows->kv_token, dt) || !stride16(rows->kv_head, dt)) return SC_ERR_INVALID_ARG;
    if (rows->q != nullptr && (!stride16(rows->q_token, dt) || !stride16(rows->q_head, dt) || !stride16(rows->qo_token, dt) || !stride16(rows->qo_head, dt)))
        return SC_ERR_INVALID_ARG;
    PagedAppendArgs a;
    a.cache = *cache; a.rows = *rows; a.dt = dt; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.T = T; a.d = d; a.flags = flags; a.status = status;
    if (rows->rot_dim == 0) a.rows.inv_freq = nullptr;
    return launch_paged_append(a, (cudaStream_t)stream) == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

size_t sc_paged_decode_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t d) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0) return 256;
    return paged_decode_ws_bytes();
}

sc_status sc_paged_decode_attn(const sc_paged_cache* cache, const void* q, sc_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                               const int32_t* lens, float scale, uint32_t flags, void* out, void* workspace, size_t workspace_bytes,
                               int32_t* status, void* stream) {
    sc_status s = check_shape(dt, B, Hq, Hkv, d);
    if (s == SC_OK) s = check_tables(cache, Hkv);
    if (s == SC_OK) s = check_pool(cache, dt, d);
    if (s != SC_OK) return s;
    if (!(scale == scale) || scale < 0.f || (flags & ~SC_FLAG_GENERIC)) return SC_ERR_INVALID_ARG;
    const int64_t heads = (int64_t)B * Hkv * div_up(Hq / Hkv, 4);
    if (heads * (((int64_t)cache->max_pages * cache->page_size + 63) / 64 * 4 + 4) > 0x7fffffff) return SC_ERR_UNSUPPORTED;   // 16-row tiles, in fours, and four more
    if (B == 0) return SC_OK;
    if (!q || !out || !lens || !workspace) return SC_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return SC_ERR_INVALID_ARG;
    if (workspace_bytes < sc_paged_decode_workspace_bytes(B, Hq, Hkv, d)) return SC_ERR_INVALID_ARG;
    PagedDecodeArgs a;
    a.cache = *cache; a.q = q; a.dt = dt; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.lens = lens; a.scale = scale; a.out = out;
    a.ws = workspace; a.status = status;
    cudaError_t e;
    if (!(flags & SC_FLAG_GENERIC) && paged_decode_mma_supported(a)) e = launch_paged_decode_mma(a, (cudaStream_t)stream);
    else e = launch_paged_decode_generic(a, (cudaStream_t)stream);
    return e == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

sc_status sc_paged_select(const sc_paged_cache* cache, const void* q, sc_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                          const int32_t* lens, int32_t keep, int32_t n_first, int32_t n_last, int32_t* sel_table, int32_t* sel_len,
                          int32_t* status, void* stream) {
    sc_status s = check_shape(dt, B, Hq, Hkv, d);
    if (s == SC_OK) s = check_tables(cache, Hkv);
    if (s != SC_OK) return s;
    if (keep < 1 || n_first < 0 || n_last < 1 || (int64_t)n_first + n_last > keep) return SC_ERR_INVALID_ARG;
    if ((int64_t)keep * cache->page_size > 0x7fffffff) return SC_ERR_INVALID_ARG;   // no table of that length could be read
    if (cache->max_pages > SC_SELECT_MAX_PAGES) return SC_ERR_UNSUPPORTED;
    if (B == 0) return SC_OK;
    if (!q || !lens || !sel_table || !sel_len) return SC_ERR_INVALID_ARG;
    if (cache->num_pages > 0 && (!cache->k_min || !cache->k_max)) return SC_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(cache->k_min) || !aligned16(cache->k_max)) return SC_ERR_INVALID_ARG;
    PagedSelectArgs a;
    a.cache = *cache; a.q = q; a.dt = dt; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.lens = lens; a.keep = keep; a.n_first = n_first;
    a.n_last = n_last; a.sel_table = sel_table; a.sel_len = sel_len; a.status = status;
    return launch_paged_select(a, (cudaStream_t)stream) == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

}  // extern "C"
