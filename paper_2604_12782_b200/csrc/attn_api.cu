// Host side of the calls around the paged key/value cache: validation, workspace layout, launches.
#include <math.h>

#include <algorithm>
#include <utility>

#include "../../include/osc.h"
#include "common.cuh"

namespace osc {

static osc_status check_cache(const osc_kv_cache_t* c) {
    if (!c) return fail(OSC_ERR_INVALID_ARG, "cache is null");
    if (c->n_pages < 0 || c->page_size < 1 || c->n_heads < 1)
        return fail(OSC_ERR_INVALID_ARG, "cache: n_pages = %d, page_size = %d, n_heads = %d", c->n_pages, c->page_size, c->n_heads);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(OSC_ERR_SHAPE, "cache: head_dim = %d, must be 64 or 128", c->head_dim);
    if ((int64_t)c->n_pages * c->page_size > 0x7FFFFFFFll)
        return fail(OSC_ERR_SHAPE, "cache: n_pages * page_size = %lld passes 2^31 - 1", (long long)c->n_pages * c->page_size);
    if (c->n_pages > 0 && (!c->k || !c->v)) return fail(OSC_ERR_INVALID_ARG, "cache: null device pointer");
    if ((c->n_pages > 1 && c->page_stride < c->head_dim) || (c->page_size > 1 && c->token_stride < c->head_dim) ||
        (c->n_heads > 1 && c->head_stride < c->head_dim))
        return fail(OSC_ERR_SHAPE, "cache: a stride is smaller than head_dim = %d", c->head_dim);
    if (c->page_stride % 8 || c->token_stride % 8 || c->head_stride % 8 || !aligned16(c->k) || !aligned16(c->v))
        return fail(OSC_ERR_ALIGN, "cache: k and v must be 16-byte aligned, strides multiples of 8");
    return OSC_OK;
}

// A matrix in memory: `rows` pieces of `width` bytes, `ld` >= width bytes from one to the next; it ends in front of `end` (which stops
// at the end of the address space, as strides are the caller's).
struct ByteRows {
    uint64_t at, end;
    int64_t rows, ld, width;
};
static ByteRows bytes_of(const void* p, int64_t rows, int64_t ld, int64_t width, int item) {
    ByteRows b = {reinterpret_cast<uintptr_t>(p), 0, rows, 0, 0};
    if (rows < 1 || width < 1) return b;
    uint64_t span = 0;
    b.width = width * item;
    bool over = __builtin_mul_overflow(ld, (int64_t)item, &b.ld);
    if (over) b.ld = INT64_MAX;
    over &= rows > 1;
    over |= rows > 1 && __builtin_mul_overflow((uint64_t)(rows - 1), (uint64_t)b.ld, &span);
    over |= __builtin_add_overflow(span, (uint64_t)b.width, &span) || __builtin_add_overflow(b.at, span, &b.end);
    if (over) b.end = ~0ull;
    return b;
}
// Whether two matrices that reach into one another share a byte.  Rows of one may lie in the gaps between the other's rows.
static bool rows_cross(const ByteRows& a, const ByteRows& b) {   // b begins inside a
    if (a.rows == 1 && b.rows == 1) return true;
    // b's rows as places on a's grid
    const __int128 ld = a.rows > 1 ? a.ld : b.ld, ldb = b.rows > 1 ? b.ld : ld, from0 = b.at - a.at;
    if (ld == ldb) {     // b's first row begins at byte c of a row of a's grid, and reaches the next one (which is there: b begins before a ends) or not
        const __int128 c = from0 % ld;
        return c < a.width || c + b.width > ld;
    }
    for (__int128 i = 0; i < b.rows; ++i) {      // a's first row that ends behind the beginning of b's
        const __int128 from = from0 + i * ldb, r = from < a.width ? 0 : (from - a.width) / ld + 1;
        if (r < a.rows && r * ld < from + b.width) return true;
    }
    return false;
}
static bool rows_meet(const ByteRows& a, const ByteRows& b) {
    if (a.end <= b.at || b.end <= a.at) return false;       // (also where one is empty: its end is 0)
    return a.at <= b.at ? rows_cross(a, b) : rows_cross(b, a);
}

// bf16 tensor map of 3 or 4 dimensions, boxes of 64 channels, 128-byte swizzle, zeros outside.  strides in elements.
static osc_status encode_heads(CUtensorMap* tm, const void* base, int rank, const int64_t* dims, const int64_t* strides, const int* box,
                               const char* what) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return fail(OSC_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    cuuint64_t gdim[4], gstr[3];
    cuuint32_t gbox[4], estr[4] = {1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) {
        gdim[i] = (cuuint64_t)dims[i];
        gbox[i] = (cuuint32_t)box[i];
        if (i) gstr[i - 1] = (cuuint64_t)(dims[i] > 1 ? strides[i] : dims[0]) * 2;
    }
    CUresult r = fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), gdim, gstr, gbox, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(OSC_ERR_CUDA, "cuTensorMapEncodeTiled(%s) failed with code %d", what, (int)r);
    return OSC_OK;
}

struct AttnLayout {
    size_t few_start, wide_start, share, cut[2], seg, tok_req, part, ml, total;
};
static AttnLayout attn_layout(int T, int n_q, int D, int R, int P) {
    AttnLayout l;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    const size_t S = (size_t)R + P;
    // rows of partial results; rows with two sources exist only where there are prefixes
    const size_t rows = AT_FEW_SLOTS + AT_WIDE_SLOTS + (P ? 2 * (size_t)T * n_q : 0);
    l.few_start = take((S + 1) * 4);
    l.wide_start = take((S + 1) * 4);
    l.share = take(12);
    l.cut[0] = take((size_t)AT_FEW_CTAS * sizeof(CutUnit));
    l.cut[1] = take((size_t)AT_WIDE_CTAS * sizeof(CutUnit));
    l.seg = take(S * sizeof(Segment));
    l.tok_req = take(P ? (size_t)T * 4 : 0);
    l.part = take(rows * D * 4);
    l.ml = take(rows * 8);
    l.total = at;
    return l;
}

}  // namespace osc

using namespace osc;

extern "C" {

osc_status osc_kv_slots(const int32_t* cached, const int32_t* fresh, const int32_t* base, int R, int page_size,
                        const int32_t* free_pages, int n_free, int32_t* table, int cols, int64_t ld_table, int T,
                        int32_t* row_off, int32_t* kv_len, int32_t* slots, int32_t* positions, int32_t* taken, void* stream) {
    if (R < 0 || T < 0 || n_free < 0 || cols < 0) return fail(OSC_ERR_INVALID_ARG, "R = %d, T = %d, n_free = %d, cols = %d", R, T, n_free, cols);
    if (page_size < 1) return fail(OSC_ERR_SHAPE, "page_size = %d", page_size);
    if (!row_off || !taken || (T > 0 && (!slots || !positions)) || (n_free > 0 && !free_pages) ||
        (R > 0 && (!cached || !fresh || !kv_len)) || (R > 0 && cols > 0 && !table))
        return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    if (R > 1 && ld_table < cols) return fail(OSC_ERR_SHAPE, "ld_table = %lld < cols = %d", (long long)ld_table, cols);
    // Every CTA reads all lengths for itself, so nothing that is written may lie on them, nor on one another.
    const struct { const int32_t* p; int64_t n; const char* name; } buf[10] = {
        {row_off, (int64_t)R + 1, "row_off"}, {kv_len, R, "kv_len"}, {slots, T, "slots"}, {positions, T, "positions"}, {taken, 1, "taken"},
        {table, R > 0 ? (R - 1) * ld_table + cols : 0, "table"}, {cached, R, "cached"}, {fresh, R, "fresh"}, {base, base ? R : 0, "base"},
        {free_pages, n_free, "free_pages"}};
    for (int i = 0; i < 6; ++i)
        for (int j = i + 1; j < 10; ++j)
            if (buf[i].n > 0 && buf[j].n > 0 && buf[i].p < buf[j].p + buf[j].n && buf[j].p < buf[i].p + buf[i].n)
                return fail(OSC_ERR_INVALID_ARG, "%s overlaps %s", buf[i].name, buf[j].name);
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    KvSlotsArgs a = {};
    a.cached = cached; a.fresh = fresh; a.base = base; a.free_pages = free_pages; a.table = table; a.ld_table = ld_table;
    a.row_off = row_off; a.kv_len = kv_len; a.slots = slots; a.positions = positions; a.taken = taken;
    a.R = R; a.page = page_size; a.n_free = n_free; a.cols = cols; a.T = T;
    cudaError_t e = launch_kv_slots(a, di.num_sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "kv_slots_kernel");
    return OSC_OK;
}

osc_status osc_qk_norm_rope(const void* QKV, int T, int64_t ld, int n_q, const osc_kv_cache_t* cache, const void* gamma_q,
                            const void* gamma_k, float eps, const osc_rope_t* rope, const int32_t* positions, int64_t ld_pos,
                            const int32_t* slots, void* Q, int64_t ldq, void* stream) {
    if (T < 0 || n_q < 1) return fail(OSC_ERR_INVALID_ARG, "T = %d, n_q = %d", T, n_q);
    if (osc_status s = check_cache(cache)) return s;
    if (!rope) return fail(OSC_ERR_INVALID_ARG, "rope is null");
    const int D = cache->head_dim;
    if (rope->rot_dim < 16 || rope->rot_dim % 16 || rope->rot_dim > D)
        return fail(OSC_ERR_SHAPE, "rot_dim = %d must be a multiple of 16 within head_dim = %d", rope->rot_dim, D);
    if (rope->axes < 1 || rope->axes > 3) return fail(OSC_ERR_INVALID_ARG, "axes = %d outside 1..3", rope->axes);
    if ((int64_t)n_q + 2ll * cache->n_heads > 65536) return fail(OSC_ERR_SHAPE, "n_q = %d, n_heads = %d: too many heads", n_q, cache->n_heads);
    if (T == 0) return OSC_OK;
    if (!QKV || !Q || !positions || !rope->inv_freq) return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    const int64_t width = ((int64_t)n_q + 2 * cache->n_heads) * D;
    if (ld < width || ldq < (int64_t)n_q * D || (rope->axes > 1 && ld_pos < T))
        return fail(OSC_ERR_SHAPE, "ld = %lld < %lld, ldq = %lld < %lld or ld_pos = %lld < T", (long long)ld, (long long)width, (long long)ldq,
                    (long long)n_q * D, (long long)ld_pos);
    if (ld % 8 || ldq % 8 || !aligned16(QKV) || !aligned16(Q) || !aligned16(gamma_q) || !aligned16(gamma_k))
        return fail(OSC_ERR_ALIGN, "QKV, Q, gamma_q and gamma_k must be 16-byte aligned, ld and ldq multiples of 8");
    if (cache->n_pages > 0 && cache->k == cache->v) return fail(OSC_ERR_INVALID_ARG, "cache: keys and values would be written to the same place");
    if (!(Q == QKV && (T == 1 || ldq == ld)) && rows_meet(bytes_of(QKV, T, ld, width, 2), bytes_of(Q, T, ldq, (int64_t)n_q * D, 2)))
        return fail(OSC_ERR_INVALID_ARG, "Q overlaps QKV and is not QKV itself with ldq = ld");
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    QkNormRopeArgs a = {};
    a.qkv = static_cast<const uint16_t*>(QKV); a.ld = ld;
    a.gamma_q = static_cast<const uint16_t*>(gamma_q); a.gamma_k = static_cast<const uint16_t*>(gamma_k);
    a.inv_freq = rope->inv_freq; a.axis = rope->axis; a.positions = positions; a.ld_pos = ld_pos;
    a.q = static_cast<uint16_t*>(Q); a.ldq = ldq;
    a.k = static_cast<uint16_t*>(cache->k); a.v = static_cast<uint16_t*>(cache->v);
    a.page_stride = cache->page_stride; a.token_stride = cache->token_stride; a.head_stride = cache->head_stride;
    a.slots = slots; a.eps = eps; a.scale = rope->scale;
    a.T = T; a.Hq = n_q; a.Hk = cache->n_heads; a.rot = rope->rot_dim; a.axes = rope->axes; a.page = cache->page_size; a.n_pages = cache->n_pages;
    cudaError_t e = launch_qk_norm_rope(a, D, rope->interleaved != 0, di.num_sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "qk_norm_rope_kernel");
    return OSC_OK;
}

static osc_status check_attention_sizes(int T, int n_q, int D, int R, int P) {
    if (T < 0 || n_q < 1 || R < 0 || P < 0) return fail(OSC_ERR_INVALID_ARG, "T = %d, n_q = %d, R = %d, P = %d", T, n_q, R, P);
    if (D != 64 && D != 128) return fail(OSC_ERR_SHAPE, "head_dim = %d, must be 64 or 128", D);
    if (n_q > 65536 || (int64_t)R + P > 0x3FFFFFFF) return fail(OSC_ERR_SHAPE, "n_q = %d, R = %d, P = %d: too many", n_q, R, P);
    return OSC_OK;
}

osc_status osc_paged_attention_workspace_bytes(int T, int n_q, int head_dim, int R, int P, size_t* bytes) {
    if (!bytes) return fail(OSC_ERR_INVALID_ARG, "bytes is null");
    if (osc_status s = check_attention_sizes(T, n_q, head_dim, R, P)) return s;
    *bytes = attn_layout(T, n_q, head_dim, R, P).total;
    return OSC_OK;
}

osc_status osc_paged_attention(const void* Q, int T, int64_t ldq, int n_q, const osc_kv_cache_t* cache, int R,
                               const int32_t* row_off, const int32_t* kv_len, const int32_t* table, int cols, int64_t ld_table,
                               int P, const int32_t* group_off, const int32_t* prefix_len, const int32_t* prefix_table,
                               int prefix_cols, int64_t ld_prefix, int max_new, float scale, void* O, int64_t ldo, float* lse,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (osc_status s = check_cache(cache)) return s;
    const int D = cache->head_dim;
    if (osc_status s = check_attention_sizes(T, n_q, D, R, P)) return s;
    if (n_q % cache->n_heads || n_q / cache->n_heads > 128)
        return fail(OSC_ERR_SHAPE, "n_q = %d must be a multiple of n_heads = %d, at most 128 times it", n_q, cache->n_heads);
    if (cache->page_size < 16 || (cache->page_size & (cache->page_size - 1)))
        return fail(OSC_ERR_SHAPE, "page_size = %d must be a power of two of at least 16", cache->page_size);
    if (cols < 0 || (P > 0 && prefix_cols < 0) || max_new < 0)
        return fail(OSC_ERR_INVALID_ARG, "cols = %d, prefix_cols = %d, max_new = %d", cols, prefix_cols, max_new);
    if (!(scale > 0.0f) || !(scale < INFINITY)) return fail(OSC_ERR_INVALID_ARG, "scale = %g must be positive and finite", (double)scale);
    if (T == 0 || R == 0) return OSC_OK;
    if (!Q || !O || !row_off || !kv_len || (cols > 0 && !table) || !workspace) return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    if (P > 0 && (!group_off || !prefix_len || (prefix_cols > 0 && !prefix_table)))
        return fail(OSC_ERR_INVALID_ARG, "null device pointer of a shared prefix");
    if ((R > 1 && ld_table < cols) || (P > 1 && ld_prefix < prefix_cols))
        return fail(OSC_ERR_SHAPE, "ld_table = %lld < cols = %d or ld_prefix = %lld < prefix_cols = %d", (long long)ld_table, cols,
                    (long long)ld_prefix, prefix_cols);
    if (ldq < (int64_t)n_q * D || ldo < (int64_t)n_q * D)
        return fail(OSC_ERR_SHAPE, "ldq = %lld, ldo = %lld < n_q * head_dim = %lld", (long long)ldq, (long long)ldo, (long long)n_q * D);
    if (ldq % 8 || ldo % 8 || !aligned16(Q) || !aligned16(O) || !aligned16(workspace))
        return fail(OSC_ERR_ALIGN, "Q, O and workspace must be 16-byte aligned, ldq and ldo multiples of 8");
    // Counts of tiles and of rows are ints on the device.  The line cannot hold more than every request's units over all the keys its
    // table names (16 keys and 16 rows to a tile at the least), nor more than that of all rows over the prefix tables.
    const int64_t own_keys = (int64_t)cols * cache->page_size, front_keys = P ? (int64_t)prefix_cols * cache->page_size : 0;
    const int64_t few_units = ((int64_t)T * (n_q / cache->n_heads)) / AT_FEW_ROWS + (int64_t)R + P;
    const int64_t wide_units = few_units / 8 + (int64_t)R + P;
    const int hw = cache->n_heads % 4 == 0 ? 4 : cache->n_heads % 2 == 0 ? 2 : 1;
    const double most_few = (double)few_units * (cache->n_heads / hw) * (std::max(own_keys, front_keys) / (64.0 / hw) + 1.0);
    const double most_wide = (double)wide_units * cache->n_heads * ((own_keys + front_keys) / 128.0 + 2.0 + WideUnits::LEAD);
    const double most_request = ((double)R + P) * (cache->n_heads / hw) * (std::max(own_keys, front_keys) / (64.0 / hw) + 1.0);
    if (own_keys > 0x20000000 || front_keys > 0x20000000)
        return fail(OSC_ERR_SHAPE, "table columns hold %lld / %lld keys, at most 2^29 are supported", (long long)own_keys, (long long)front_keys);
    if (most_wide >= 2147483648.0 || most_request >= 2147483648.0 || (cache->n_pages == 0 && most_few >= 2147483648.0) || (int64_t)T * n_q > 0x20000000)
        return fail(OSC_ERR_SHAPE, "T = %d, R = %d, P = %d over up to %lld keys: too many tiles", T, R, P, (long long)(own_keys + front_keys));
    const AttnLayout l = attn_layout(T, n_q, D, R, P);
    if (workspace_bytes < l.total) return fail(OSC_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, l.total);
    // What is written may lie on nothing else: other CTAs still read it.
    const int64_t width = (int64_t)n_q * D;
    const struct { ByteRows b; const char* name; } buf[10] = {
        {bytes_of(O, T, ldo, width, 2), "O"}, {bytes_of(lse, lse ? 1 : 0, 0, (int64_t)T * n_q, 4), "lse"},
        {bytes_of(workspace, 1, 0, (int64_t)l.total, 1), "the workspace"}, {bytes_of(Q, T, ldq, width, 2), "Q"},
        {bytes_of(row_off, 1, 0, (int64_t)R + 1, 4), "row_off"}, {bytes_of(kv_len, 1, 0, R, 4), "kv_len"}, {bytes_of(table, R, ld_table, cols, 4), "table"},
        {bytes_of(group_off, P ? 1 : 0, 0, (int64_t)P + 1, 4), "group_off"}, {bytes_of(prefix_len, P ? 1 : 0, 0, P, 4), "prefix_len"},
        {bytes_of(prefix_table, P, ld_prefix, prefix_cols, 4), "prefix_table"}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 10; ++j)
            if (rows_meet(buf[i].b, buf[j].b)) return fail(OSC_ERR_INVALID_ARG, "%s overlaps %s", buf[i].name, buf[j].name);
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    AttnWideArgs w = {};
    AttnArgs& a = w.a;
    a.q = static_cast<const uint16_t*>(Q); a.ldq = ldq; a.o = static_cast<uint16_t*>(O); a.ldo = ldo; a.lse = lse;
    // copies of absent pages read nothing, but are given an address: that of Q where there is no cache
    a.k = static_cast<const uint16_t*>(cache->n_pages ? cache->k : Q); a.v = static_cast<const uint16_t*>(cache->n_pages ? cache->v : Q);
    a.page_stride = cache->page_stride; a.token_stride = cache->token_stride; a.head_stride = cache->head_stride;
    a.row_off = row_off; a.kv_len = kv_len; a.table = table; a.ld_table = ld_table; a.cols = cols;
    a.group_off = group_off; a.prefix_len = prefix_len; a.ptable = prefix_table; a.ld_ptable = ld_prefix; a.pcols = P ? prefix_cols : 0;
    a.T = T; a.Hq = n_q; a.Hk = cache->n_heads; a.G = n_q / cache->n_heads; a.tpt = AT_WIDE_TILE / a.G; a.inv_g = (65536 + a.G - 1) / a.G; a.head_dim = D; a.R = R; a.P = P; a.n_pages = cache->n_pages;
    while ((1 << a.page_shift) < cache->page_size) ++a.page_shift;
    a.scale_log2 = scale * 1.44269504088896341f;
    a.few_hw = hw;
    a.wide_ctas = di.num_sms < AT_WIDE_CTAS ? di.num_sms : AT_WIDE_CTAS;
    // Up to 16 rows per key/value head a request is one unit of the few-row kernel, whatever the rest of the step is.  The tcgen05
    // kernel is launched where a segment may have more: a shared prefix, or requests with more new tokens than that.
    // (Nor may the 16-row units of a step whose max_new is wrong be too many to count.)
    const bool wide = a.n_pages > 0 && (P > 0 || max_new == 0 || (int64_t)max_new * a.G > AT_FEW_ROWS || most_few >= 2147483648.0);
    a.few_ctas = std::min(di.num_sms * (wide ? 4 : 2), AT_FEW_CTAS);
    a.wide_min_rows = wide ? AT_FEW_ROWS + 1 : 0x7FFFFFFF;
    if (wide) {
        const int64_t qd[3] = {D, n_q, T}, qs[3] = {1, D, ldq};
        const int qb[3] = {64, a.G, a.tpt};
        const int64_t kd[4] = {D, cache->page_size, cache->n_heads, cache->n_pages};
        const int64_t ks[4] = {1, cache->token_stride, cache->head_stride, cache->page_stride};
        const int kb[4] = {64, cache->page_size < AT_WIDE_KEYS ? cache->page_size : AT_WIDE_KEYS, 1, 1};
        if (osc_status s = encode_heads(&w.tm_q, Q, 3, qd, qs, qb, "Q")) return s;
        if (osc_status s = encode_heads(&w.tm_k, cache->k, 4, kd, ks, kb, "K")) return s;
        if (osc_status s = encode_heads(&w.tm_v, cache->v, 4, kd, ks, kb, "V")) return s;
    }
    a.plan.few_start = reinterpret_cast<int32_t*>(ws + l.few_start);
    a.plan.wide_start = reinterpret_cast<int32_t*>(ws + l.wide_start);
    a.plan.share = reinterpret_cast<int32_t*>(ws + l.share);
    for (int i = 0; i < 2; ++i) a.plan.cut[i] = reinterpret_cast<CutUnit*>(ws + l.cut[i]);
    a.plan.seg = reinterpret_cast<Segment*>(ws + l.seg);
    a.plan.tok_req = reinterpret_cast<int32_t*>(ws + l.tok_req);
    a.part = reinterpret_cast<float*>(ws + l.part);
    a.ml = reinterpret_cast<float2*>(ws + l.ml);
    cudaError_t e = launch_attn(w, D, wide, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "attention kernels");
    return OSC_OK;
}

}  // extern "C"
