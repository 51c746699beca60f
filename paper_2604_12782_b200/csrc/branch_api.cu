// Host side of the calls for requests with more than one continuation: moves in the paged cache, scores of tokens.
#include <stdlib.h>

#include <algorithm>

#include "../../include/osc.h"
#include "common.cuh"

namespace osc {

// Layers of one shape, at most KV_LAYERS of them from `first` on.
static osc_status check_layers(const osc_kv_cache_t* layers, int n_layers) {
    if (n_layers < 1 || !layers) return fail(OSC_ERR_INVALID_ARG, "layers is null or n_layers = %d", n_layers);
    if (osc_status s = check_cache(&layers[0])) return s;
    const osc_kv_cache_t& c = layers[0];
    if ((int64_t)c.n_heads * c.head_dim > 0x1000000) return fail(OSC_ERR_SHAPE, "cache: n_heads = %d, too many", c.n_heads);
    for (int i = 0; i < n_layers; ++i) {
        const osc_kv_cache_t& x = layers[i];
        if (x.n_pages != c.n_pages || x.page_size != c.page_size || x.n_heads != c.n_heads || x.head_dim != c.head_dim ||
            x.page_stride != c.page_stride || x.token_stride != c.token_stride || x.head_stride != c.head_stride)
            return fail(OSC_ERR_SHAPE, "layer %d has another shape or other strides than layer 0", i);
        if (x.n_pages > 0 && (!x.k || !x.v)) return fail(OSC_ERR_INVALID_ARG, "layer %d: null device pointer", i);
        if (!aligned16(x.k) || !aligned16(x.v)) return fail(OSC_ERR_ALIGN, "layer %d: k and v must be 16-byte aligned", i);
        if (x.n_pages > 0 && x.k == x.v) return fail(OSC_ERR_INVALID_ARG, "layer %d: keys and values are the same place", i);
    }
    return OSC_OK;
}

// Keys or values that two layers share would be moved twice, the second time from places that are overwritten already.  A table of addresses, a quarter full at
// most: 36 layers 0.3 us.
static osc_status check_planes_apart(const osc_kv_cache_t* layers, int n_layers) {
    if (layers[0].n_pages == 0) return OSC_OK;
    int bits = 3;
    while ((int64_t)1 << bits < 8ll * n_layers) ++bits;
    const size_t mask = ((size_t)1 << bits) - 1;
    uintptr_t* table = static_cast<uintptr_t*>(calloc(mask + 1, sizeof(uintptr_t)));
    if (!table) return fail(OSC_ERR_INVALID_ARG, "n_layers = %d: no memory on the host", n_layers);
    int again = -1;
    for (int i = 0; i < 2 * n_layers && again < 0; ++i) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(i & 1 ? layers[i / 2].v : layers[i / 2].k);
        size_t at = (size_t)((p >> 4) * 0x9E3779B97F4A7C15ull >> (64 - bits));
        while (table[at] && table[at] != p) at = (at + 1) & mask;
        if (table[at]) again = i;
        table[at] = p;
    }
    free(table);
    if (again >= 0) return fail(OSC_ERR_INVALID_ARG, "layer %d: %s are another layer's too", again / 2, again & 1 ? "values" : "keys");
    return OSC_OK;
}

static KvPlanes planes_of(const osc_kv_cache_t* layers, int n) {
    KvPlanes l;
    const osc_kv_cache_t& c = layers[0];
    for (int i = 0; i < n; ++i) {
        l.p[2 * i] = static_cast<uint4*>(layers[i].k);
        l.p[2 * i + 1] = static_cast<uint4*>(layers[i].v);
    }
    l.page_stride = c.page_stride / 8;
    l.token_stride = c.token_stride / 8;
    l.head_stride = c.head_stride / 8;
    l.n_pages = c.n_pages;
    l.page = c.page_size;
    l.head_shift = c.head_dim == 128 ? 4 : 3;
    l.row = c.n_heads << l.head_shift;
    l.planes = 2 * n;
    return l;
}

struct NamedRows {
    ByteRows b;
    const char* name;
};
// What is written (the first `written` buffers) may lie on nothing else.
static osc_status check_apart(const NamedRows* buf, int n, int written) {
    for (int i = 0; i < written; ++i)
        for (int j = i + 1; j < n; ++j)
            if (rows_meet(buf[i].b, buf[j].b)) return fail(OSC_ERR_INVALID_ARG, "%s overlaps %s", buf[i].name, buf[j].name);
    return OSC_OK;
}
static ByteRows ints(const void* p, int64_t n) { return bytes_of(p, p ? 1 : 0, 0, n, 4); }

}  // namespace osc

using namespace osc;

extern "C" {

osc_status osc_kv_compact(const osc_kv_cache_t* layers, int n_layers, int R, const int32_t* row_off, const int32_t* kv_len, const int32_t* table,
                          int cols, int64_t ld_table, const int32_t* keep, int keep_cols, int64_t ld_keep, const int32_t* n_keep,
                          int32_t* new_len, void* stream) {
    if (osc_status s = check_layers(layers, n_layers)) return s;
    if (R < 0 || cols < 0 || keep_cols < 0) return fail(OSC_ERR_INVALID_ARG, "R = %d, cols = %d, keep_cols = %d", R, cols, keep_cols);
    if (R > (1 << 20)) return fail(OSC_ERR_SHAPE, "R = %d: at most 2^20 requests", R);
    if (R == 0) return OSC_OK;
    if (!row_off || !kv_len || !n_keep || !new_len || (cols > 0 && !table) || (keep_cols > 0 && !keep))
        return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    if (R > 1 && (ld_table < cols || ld_keep < keep_cols))
        return fail(OSC_ERR_SHAPE, "ld_table = %lld < cols = %d or ld_keep = %lld < keep_cols = %d", (long long)ld_table, cols, (long long)ld_keep, keep_cols);
    const NamedRows buf[6] = {{ints(new_len, R), "new_len"}, {ints(row_off, (int64_t)R + 1), "row_off"}, {ints(kv_len, R), "kv_len"},
                              {bytes_of(table, cols ? R : 0, ld_table, cols, 4), "table"}, {bytes_of(keep, keep_cols ? R : 0, ld_keep, keep_cols, 4), "keep"},
                              {ints(n_keep, R), "n_keep"}};
    if (osc_status s = check_apart(buf, 6, 1)) return s;
    if (osc_status s = check_planes_apart(layers, n_layers)) return s;
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    for (int at = 0; at < n_layers; at += KV_LAYERS) {
        KvCompactArgs a = {};
        a.l = planes_of(layers + at, std::min(n_layers - at, KV_LAYERS));
        a.row_off = row_off; a.kv_len = kv_len; a.table = table; a.ld_table = ld_table; a.keep = keep; a.ld_keep = ld_keep; a.n_keep = n_keep;
        a.new_len = new_len; a.R = R; a.cols = cols; a.keep_cols = keep_cols;
        cudaError_t e = launch_kv_compact(a, at == 0, di.num_sms, static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return cuda_fail(e, "kv_compact_kernel");
    }
    return OSC_OK;
}

osc_status osc_kv_copy_pages(const osc_kv_cache_t* layers, int n_layers, const int32_t* from, const int32_t* to, const int32_t* used, int n,
                             void* stream) {
    if (osc_status s = check_layers(layers, n_layers)) return s;
    if (n < 0) return fail(OSC_ERR_INVALID_ARG, "n = %d", n);
    if (n > (1 << 22)) return fail(OSC_ERR_SHAPE, "n = %d: at most 2^22 pages", n);
    if (n == 0 || layers[0].n_pages == 0) return OSC_OK;
    if (!from || !to) return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    for (int at = 0; at < n_layers; at += KV_LAYERS) {
        KvCopyArgs a = {};
        a.l = planes_of(layers + at, std::min(n_layers - at, KV_LAYERS));
        a.from = from; a.to = to; a.used = used; a.n = n;
        cudaError_t e = launch_kv_copy_pages(a, di.num_sms, static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return cuda_fail(e, "kv_copy_pages_kernel");
    }
    return OSC_OK;
}

osc_status osc_kv_trim(const int32_t* from_len, const int32_t* to_len, int R, int page_size, int32_t* table, int cols, int64_t ld_table,
                       int32_t* refs, int n_pages, int32_t* freed, int32_t* n_freed, void* stream) {
    if (R < 0 || cols < 0 || n_pages < 0) return fail(OSC_ERR_INVALID_ARG, "R = %d, cols = %d, n_pages = %d", R, cols, n_pages);
    if (page_size < 1) return fail(OSC_ERR_SHAPE, "page_size = %d", page_size);
    if (n_pages > TRIM_CLUSTER * (TRIM_MAX_WORDS - 1) * 32) return fail(OSC_ERR_SHAPE, "n_pages = %d: at most 12 million", n_pages);
    if (!n_freed || (n_pages > 0 && !freed) || (R > 0 && (!from_len || !to_len)) || (R > 0 && cols > 0 && !table))
        return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    if (R > 1 && ld_table < cols) return fail(OSC_ERR_SHAPE, "ld_table = %lld < cols = %d", (long long)ld_table, cols);
    const NamedRows buf[6] = {{ints(n_freed, 1), "n_freed"}, {ints(freed, n_pages), "freed"}, {bytes_of(table, cols ? R : 0, ld_table, cols, 4), "table"},
                              {ints(refs, n_pages), "refs"}, {ints(from_len, R), "from_len"}, {ints(to_len, R), "to_len"}};
    if (osc_status s = check_apart(buf, 6, 4)) return s;
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    KvTrimArgs a = {};
    a.from = from_len; a.to = to_len; a.table = table; a.ld_table = ld_table; a.refs = refs; a.freed = freed; a.n_freed = n_freed;
    a.R = R; a.page = page_size; a.cols = cols; a.n_pages = n_pages;
    cudaError_t e = launch_kv_trim(a, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "kv_trim_kernel");
    return OSC_OK;
}

osc_status osc_kv_fork(const int32_t* src, const int32_t* dst, int n, int32_t* len, int R, int page_size, const int32_t* free_pages, int n_free,
                       int32_t* table, int cols, int64_t ld_table, int32_t* refs, int n_pages, int32_t* copy_from, int32_t* copy_to,
                       int32_t* copy_used, int32_t* taken, void* stream) {
    if (n < 0 || R < 0 || n_free < 0 || cols < 0 || n_pages < 0)
        return fail(OSC_ERR_INVALID_ARG, "n = %d, R = %d, n_free = %d, cols = %d, n_pages = %d", n, R, n_free, cols, n_pages);
    if (page_size < 1) return fail(OSC_ERR_SHAPE, "page_size = %d", page_size);
    if (!taken || (n > 0 && (!src || !dst || !copy_from || !copy_to || !copy_used)) || (n_free > 0 && !free_pages) || (n > 0 && R > 0 && !len) ||
        (n > 0 && R > 0 && cols > 0 && !table))
        return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    if (R > 1 && ld_table < cols) return fail(OSC_ERR_SHAPE, "ld_table = %lld < cols = %d", (long long)ld_table, cols);
    const NamedRows buf[10] = {{ints(taken, 1), "taken"}, {ints(copy_from, n), "copy_from"}, {ints(copy_to, n), "copy_to"}, {ints(copy_used, n), "copy_used"},
                               {ints(len, R), "len"}, {bytes_of(table, cols ? R : 0, ld_table, cols, 4), "table"}, {ints(refs, n_pages), "refs"},
                               {ints(src, n), "src"}, {ints(dst, n), "dst"}, {ints(free_pages, n_free), "free_pages"}};
    if (osc_status s = check_apart(buf, 10, 7)) return s;
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    KvForkArgs a = {};
    a.src = src; a.dst = dst; a.len = len; a.free_pages = free_pages; a.table = table; a.ld_table = ld_table; a.refs = refs;
    a.copy_from = copy_from; a.copy_to = copy_to; a.copy_used = copy_used; a.taken = taken;
    a.n = n; a.R = R; a.page = page_size; a.n_free = n_free; a.cols = cols; a.n_pages = n_pages;
    cudaError_t e = launch_kv_fork(a, di.num_sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "kv_fork_kernel");
    return OSC_OK;
}

osc_status osc_token_logprobs(const void* logits, int dtype, int T, int V, int64_t ld, float scale, const int32_t* ids, int n_ids, int64_t ld_ids,
                              float* logprob, float* lse, float* entropy, int top_k, int32_t* top_ids, float* top_logprobs, void* stream) {
    if (dtype != OSC_BF16 && dtype != OSC_F32) return fail(OSC_ERR_INVALID_ARG, "dtype = %d must be OSC_BF16 or OSC_F32", dtype);
    if (T < 0 || V < 1 || n_ids < 0 || top_k < 0) return fail(OSC_ERR_INVALID_ARG, "T = %d, V = %d, n_ids = %d, top_k = %d", T, V, n_ids, top_k);
    if (top_k > LP_MAX_TOP) return fail(OSC_ERR_SHAPE, "top_k = %d: at most %d", top_k, LP_MAX_TOP);
    if (V > 0x40000000) return fail(OSC_ERR_SHAPE, "V = %d: at most 2^30", V);
    if (!(scale > 0.0f) || !(scale < 1e30f)) return fail(OSC_ERR_INVALID_ARG, "scale = %g must be positive and below 1e30", (double)scale);
    if (T == 0) return OSC_OK;
    if (!logits || (n_ids > 0 && (!ids || !logprob)) || (top_k > 0 && (!top_ids || !top_logprobs))) return fail(OSC_ERR_INVALID_ARG, "null device pointer");
    if (T > 1 && (ld < V || ld_ids < n_ids)) return fail(OSC_ERR_SHAPE, "ld = %lld < V = %d or ld_ids = %lld < n_ids = %d", (long long)ld, V, (long long)ld_ids, n_ids);
    const int item = dtype == OSC_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % item) return fail(OSC_ERR_ALIGN, "logits must be aligned to an element");
    const NamedRows buf[7] = {{ints(logprob, (int64_t)T * n_ids), "logprob"}, {ints(lse, T), "lse"}, {ints(entropy, T), "entropy"},
                              {ints(top_ids, (int64_t)T * top_k), "top_ids"}, {ints(top_logprobs, (int64_t)T * top_k), "top_logprobs"},
                              {bytes_of(logits, T, ld, V, item), "logits"}, {bytes_of(ids, n_ids ? T : 0, ld_ids, n_ids, 4), "ids"}};
    if (osc_status s = check_apart(buf, 7, 5)) return s;
    DeviceInfo di;
    if (osc_status s = device_info(&di)) return s;
    LogprobArgs a = {};
    a.x = logits; a.ld = ld; a.ids = ids; a.ld_ids = ld_ids; a.logprob = logprob; a.lse = lse; a.entropy = entropy; a.top_ids = top_ids;
    a.top_logprob = top_logprobs; a.T = T; a.V = V; a.n_ids = n_ids; a.k = top_k; a.scale = scale;
    cudaError_t e = launch_token_logprobs(a, dtype == OSC_F32, di.num_sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "token_logprobs_kernel");
    return OSC_OK;
}

}  // extern "C"
