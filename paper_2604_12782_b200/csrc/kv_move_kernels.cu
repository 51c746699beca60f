// Kernels for requests with more than one continuation, around the paged key/value cache:
//   tree_mask_kernel      ancestors and positions of the tokens of drafted trees
//   kv_compact_kernel     keys and values of accepted tokens moved together behind the context, in all layers
//   kv_trim_kernel        pages given back
//   kv_fork_kernel        rows of the page table forked
//   kv_copy_pages_kernel  pages copied, in all layers
#include <algorithm>

#include "../../include/osc.h"
#include "common.cuh"

namespace osc {

__device__ __forceinline__ int clamp_row(const int32_t* row_off, int r, int T) { return min(max(row_off[r], 0), T); }

// Inclusive sum over the block; s_warp: [32] in shared memory.  `total` is the block's.
__device__ __forceinline__ long long block_scan(long long v, long long& total, long long* s_warp, int warps) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += up;
    }
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    long long before = 0;
    total = 0;
    for (int w = 0; w < warps; ++w) {
        if (w < warp) before += s_warp[w];
        total += s_warp[w];
    }
    __syncthreads();
    return v + before;
}

// largest i in [0, n) with start[i] <= x (start ascending, start[0] <= x)
__device__ __forceinline__ int search_last(const long long* start, int n, long long x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// --------------------------------------------------------------------------------------------- tree_mask
// Token i of a request has a parent p < i among the request's new tokens, or -1 (a root).  Bit m of its row says whether m is i or an
// ancestor of i; position = base + number of ancestors.  A token whose line does not end in a root, or that has no bit (from 32 * words
// on), gets no bits and position 0.
// A request's parents go through shared memory; a thread walks up from its token.  Parents come before their children, so the
// walk meets falling indices and a row's words are finished one after the other, without an array.  Latency bounds it: offsets -> parents ->
// walk -> stores, each step of a walk one shared-memory load (a chain of 1024 tokens is the longest).  26 tokens of one request 4.2 us from a CUDA graph, an empty
// launch's time; 16201 tokens of 500 requests 7.6 us, where the bytes would take 0.1.  A block for every request, not one for several, as the chain is the time.
constexpr int TREE_THREADS = 128;

struct TreeMaskArgs {
    const int32_t* parents;
    const int32_t* row_off;
    const int32_t* base;     // may be null: 0
    uint32_t* mask;
    int64_t ld_mask;
    int32_t* positions;      // may be null
    int R, T, words;
};

__global__ void __launch_bounds__(TREE_THREADS) tree_mask_kernel(const TreeMaskArgs a) {
    __shared__ int16_t s_par[32 * OSC_TREE_WORDS];
    grid_launch_dependents();
    grid_dependency_wait();
    const int cap = 32 * a.words;
    for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
        const int t0 = clamp_row(a.row_off, r, a.T), n = clamp_row(a.row_off, r + 1, a.T) - t0, known = min(n, cap);
        const int base = a.base ? a.base[r] : 0;
        for (int i = threadIdx.x; i < known; i += TREE_THREADS) {
            const int p = a.parents[t0 + i];
            s_par[i] = p >= -1 && p < i ? (int16_t)p : (int16_t)-2;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += TREE_THREADS) {
            uint32_t* row = a.mask + (int64_t)(t0 + i) * a.ld_mask;
            int depth = -1, at = i < known ? i : -2, w = a.words - 1;
            uint32_t bits = 0;
            while (at >= 0) {
                for (; w > at >> 5; --w) {           // words above the token's
                    row[w] = bits;
                    bits = 0;
                }
                bits |= 1u << (at & 31);
                ++depth;
                at = s_par[at];
            }
            if (at == -2) bits = 0;
            for (; w >= 0; --w) {
                row[w] = bits;
                bits = 0;
            }
            if (at == -2 && depth >= 0)              // the line leads nowhere: what was written of it is taken back
                for (w = 0; w < a.words; ++w) row[w] = 0;
            if (a.positions) a.positions[t0 + i] = at == -2 ? 0 : base + depth;
        }
        __syncthreads();
    }
    // rows that only fill the step up
    for (int64_t t = (a.R ? clamp_row(a.row_off, a.R, a.T) : 0) + (int64_t)blockIdx.x * TREE_THREADS + threadIdx.x; t < a.T; t += (int64_t)gridDim.x * TREE_THREADS) {
        for (int w = 0; w < a.words; ++w) a.mask[t * a.ld_mask + w] = 0;
        if (a.positions) a.positions[t] = 0;
    }
}

cudaError_t launch_tree_mask(const TreeMaskArgs& a, int num_sms, cudaStream_t st) {
    const int grid = std::max(1, std::min(std::max(a.R, a.T / 1024), num_sms * 16));
    return launch_pdl(tree_mask_kernel, dim3(grid), dim3(TREE_THREADS), 0, st, a);
}

// ---------------------------------------------------------------------------------------- moves in the cache
// Layers of one shape; their pointers travel as a kernel argument (2 KB).
constexpr int KV_LAYERS = 128;       // most of one launch
struct KvPlanes {
    uint4* p[2 * KV_LAYERS];         // keys and values of a layer next to each other
    int64_t page_stride, token_stride, head_stride;      // in units of 16 bytes
    int n_pages, page, row;          // row: 16-byte units of a token in a plane
    int head_shift;                  // log2 of the units of a head: 3 or 4
    int planes;
};

__device__ __forceinline__ int64_t unit_offset(const KvPlanes& l, int u) {
    return (int64_t)(u >> l.head_shift) * l.head_stride + (u & ((1 << l.head_shift) - 1));
}

// kv_compact: the request's new tokens lie at places ctx = kv_len - n and on; entry d of its list (indices that rise) names the token that
// goes to place ctx + d.  An index is at least its place in the list, so walking the list in order never overwrites what is still to be
// read, and neither does reading several entries ahead: a thread takes one 16-byte column of one plane (keys or values of a layer) and
// moves it for all entries, KC_FLIGHT loads at a time.  Every byte is read and written once: HBM bounds it once there is enough of it, the
// chain offsets -> list -> pages -> rows in front of the first load before that.  96 requests, 36 layers, 86 MB read and written: 21.6 us from a CUDA graph, 17 to 18 of
// them in the kernel, where the copy rate gives 13.1; one request 4.2 us.  What is left of the 96 is that chain, three trips to memory before a block's
// rows.  Three columns to a thread (26.7 us) and eight entries under way (23.6) were no better: a request accepts about three tokens, so there is little to keep under way, and
// other blocks are what hides the chain.
constexpr int KC_THREADS = 256, KC_LIST = 256, KC_FLIGHT = 4;

struct KvCompactArgs {
    KvPlanes l;
    const int32_t* row_off;
    const int32_t* kv_len;
    const int32_t* table;
    int64_t ld_table;
    const int32_t* keep;
    int64_t ld_keep;
    const int32_t* n_keep;
    int32_t* new_len;
    int R, cols, keep_cols, splits;
};

__global__ void __launch_bounds__(KC_THREADS) kv_compact_kernel(const __grid_constant__ KvCompactArgs a, bool write_len) {
    __shared__ int64_t s_from[KC_LIST], s_to[KC_LIST];
    __shared__ int s_stop, s_moved;      // first entry that ends the list, first one that moves
    grid_launch_dependents();
    grid_dependency_wait();
    const KvPlanes& l = a.l;
    const int r = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int n = max(a.row_off[r + 1] - a.row_off[r], 0);
    const int64_t ctx = (int64_t)a.kv_len[r] - n;
    const int count = min(min(max(a.n_keep[r], 0), a.keep_cols), n);
    const int32_t* keep = a.keep + (int64_t)r * a.ld_keep;
    const int32_t* pages = a.table + (int64_t)r * a.ld_table;
    auto place = [&](int64_t at) -> int64_t {
        const int64_t col = at / l.page;
        if (at < 0 || col >= a.cols) return -1;
        const int p = pages[col];
        return p >= 0 && p < l.n_pages ? p * l.page_stride + (at - col * l.page) * l.token_stride : -1;
    };
    int done = 0;
    while (true) {               // KC_LIST entries at a time
        // The list is read next to the lengths, and the pages of all its entries next to the check of their order: two trips to memory in front of the rows.
        const int d = done + threadIdx.x;
        int k = -1, last = -1;
        if (d < a.keep_cols) {
            k = keep[d];
            if (d) last = keep[d - 1];
        }
        if (threadIdx.x == 0) s_stop = s_moved = KC_LIST;
        __syncthreads();
        if (d < count) {
            if (k >= n || k <= last) atomicMin(&s_stop, (int)threadIdx.x);
            if (k != d) atomicMin(&s_moved, (int)threadIdx.x);
            s_from[threadIdx.x] = place(ctx + k);
            s_to[threadIdx.x] = place(ctx + d);
        }
        __syncthreads();
        // entries that stay where they are come first (an index above its place leaves all behind it above theirs)
        const int good = min(s_stop, min(count - done, KC_LIST)), still = min(s_moved, good);
        if (still < good)
            for (int x = split * KC_THREADS + threadIdx.x; x < l.planes * l.row; x += a.splits * KC_THREADS) {
                const int plane = x / l.row;
                uint4* base = l.p[plane] + unit_offset(l, x - plane * l.row);
                for (int i = still; i < good; i += KC_FLIGHT) {
                    uint4 v[KC_FLIGHT];
#pragma unroll
                    for (int j = 0; j < KC_FLIGHT; ++j)
                        if (i + j < good && s_from[i + j] >= 0) v[j] = base[s_from[i + j]];
#pragma unroll
                    for (int j = 0; j < KC_FLIGHT; ++j)
                        if (i + j < good && s_from[i + j] >= 0 && s_to[i + j] >= 0) base[s_to[i + j]] = v[j];
                }
            }
        done += good;
        __syncthreads();
        if (good < KC_LIST) break;
    }
    if (write_len && split == 0 && threadIdx.x == 0) a.new_len[r] = (int)(ctx + done);
}

// kv_copy_pages: the first `used` places of page from[i] to page to[i], in every plane.  A block takes a part of one page of one plane; its threads
// walk over 16-byte units, KP_FLIGHT loads at a time.  HBM: 1505 tokens of 90 forks in 36 layers, 444 MB read and written, in 65 us, the copy rate; the planes of a page are neighbours
// on the grid because their pages are the same, so that a block's three trips (pages, count, rows) overlap with its neighbours' rows.
constexpr int KP_THREADS = 256, KP_FLIGHT = 8;

struct KvCopyArgs {
    KvPlanes l;
    const int32_t* from;
    const int32_t* to;
    const int32_t* used;      // may be null: whole pages
    int n, parts;             // parts of a page
    int step_token, step_unit;     // KP_THREADS as tokens and units of a token
};

__global__ void __launch_bounds__(KP_THREADS) kv_copy_pages_kernel(const __grid_constant__ KvCopyArgs a) {
    grid_launch_dependents();
    grid_dependency_wait();
    const KvPlanes& l = a.l;
    const int plane = blockIdx.x % l.planes, rest = blockIdx.x / l.planes, part = rest % a.parts, i = rest / a.parts;
    const int from = a.from[i], to = a.to[i];
    const int used = a.used ? min(max(a.used[i], 0), l.page) : l.page;
    if (from < 0 || from >= l.n_pages || to < 0 || to >= l.n_pages || from == to) return;
    const int t0 = (int)((int64_t)used * part / a.parts), t1 = (int)((int64_t)used * (part + 1) / a.parts);
    const uint4* src = l.p[plane] + from * l.page_stride;
    uint4* dst = l.p[plane] + to * l.page_stride;
    int token = t0 + threadIdx.x / l.row, unit = threadIdx.x % l.row;
    while (token < t1) {
        uint4 v[KP_FLIGHT];
        int64_t off[KP_FLIGHT];
#pragma unroll
        for (int j = 0; j < KP_FLIGHT; ++j) {
            off[j] = token < t1 ? token * l.token_stride + unit_offset(l, unit) : -1;
            if (off[j] >= 0) v[j] = __ldcs(src + off[j]);
            token += a.step_token;
            unit += a.step_unit;
            if (unit >= l.row) { unit -= l.row; ++token; }
        }
#pragma unroll
        for (int j = 0; j < KP_FLIGHT; ++j)
            if (off[j] >= 0) dst[off[j]] = v[j];
    }
}

cudaError_t launch_kv_compact(const KvCompactArgs& args, bool write_len, int num_sms, cudaStream_t st) {
    KvCompactArgs a = args;
    // A block for every KC_THREADS columns, as long as that is no more than 16 to an SM, two to three rounds of those resident (96 / 250 / 600 requests, 86 / 207 / 160 MB: 24.4 / 54.9 / - us
    // with 6, 22.3 / 49.6 / 49.3 with 8, 21.6 / 44.4 / 36.8 with 16, 21.9 / 41.5 / 35.1 with 32, where other sizes take 6-8 % longer than with 16).
    const int most = (a.l.planes * a.l.row + KC_THREADS - 1) / KC_THREADS;
    a.splits = std::max(1, std::min(most, num_sms * 16 / std::max(a.R, 1)));
    return launch_pdl(kv_compact_kernel, dim3(a.R * a.splits), dim3(KC_THREADS), 0, st, a, write_len);
}

cudaError_t launch_kv_copy_pages(const KvCopyArgs& args, int num_sms, cudaStream_t st) {
    KvCopyArgs a = args;
    const int64_t items = (int64_t)a.n * a.l.planes;
    // enough blocks to fill the machine twice, parts of at least KP_THREADS * KP_FLIGHT units
    const int64_t most = std::max<int64_t>(1, (int64_t)a.l.page * a.l.row / (KP_THREADS * KP_FLIGHT));
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, (int64_t)num_sms * 16 / items));
    a.step_token = KP_THREADS / a.l.row;
    a.step_unit = KP_THREADS % a.l.row;
    return launch_pdl(kv_copy_pages_kernel, dim3((unsigned)(items * a.parts)), dim3(KP_THREADS), 0, st, a);
}

// ------------------------------------------------------------------------------------------------ kv_trim
// Request r gives back the pages of columns ceil(to / p) .. ceil(from / p) - 1 of its row: the entries become -1, the pages' counts of
// holders fall by one, and a page whose last holder this was is freed.  The freed pages come out in rising order, whatever order the blocks ran in.
// One cluster: the rows' columns are flattened (a scan over the requests, which every block does for itself) and shared out over all
// its threads; the bitmap of freed pages is spread over the blocks' shared memories (remote atomics), so nothing has to be cleared or kept in
// global memory; then every block lists its part behind those of lower rank.  The decrement that takes a count from 1 to 0 happens once,
// so does its bit.  (A count that was 0 or less is put back: it never reaches 1 on the way.)  Latency bounds it: 7 to 8 us for 192 rows.  One launch of one
// cluster instead of three of a grid (clear, mark, list): the bitmap is small, and a launch costs as much as the whole call.
constexpr int TRIM_CLUSTER = 8, TRIM_THREADS = 512;
constexpr int TRIM_MAX_WORDS = 48 * 1024;     // of a block's part of the bitmap: 12.5 million pages in all

struct KvTrimArgs {
    const int32_t* from;
    const int32_t* to;
    int32_t* table;
    int64_t ld_table;
    int32_t* refs;           // may be null: every page has one holder
    int32_t* freed;
    int32_t* n_freed;
    int R, page, cols, n_pages, part;     // part: words of a block's part of the bitmap
};

__device__ __forceinline__ void atom_or_cluster(uint32_t addr, uint32_t v) {
    asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

__global__ void __launch_bounds__(TRIM_THREADS) kv_trim_kernel(const KvTrimArgs a) {
    extern __shared__ uint32_t s_bits[];
    __shared__ long long s_start[TRIM_THREADS], s_warp[32];
    __shared__ int s_col[TRIM_THREADS];
    __shared__ uint32_t s_count[TRIM_CLUSTER];
    grid_launch_dependents();
    const int tid = threadIdx.x, rank = (int)cluster_ctarank();
    for (int w = tid; w < a.part; w += TRIM_THREADS) s_bits[w] = 0;
    const uint32_t bits = smem_u32(s_bits), counts = smem_u32(s_count);
    grid_dependency_wait();
    __syncwarp();
    cluster_sync_all();      // all parts are clear
    for (int r0 = 0; r0 < a.R; r0 += TRIM_THREADS) {
        const int nr = min(TRIM_THREADS, a.R - r0);
        long long own = 0, total;
        if (tid < nr) {
            const long long p = a.page, from = max(a.from[r0 + tid], 0), to = max(a.to[r0 + tid], 0);
            const long long c0 = (to + p - 1) / p, c1 = min((from + p - 1) / p, (long long)a.cols);
            own = max(c1 - c0, 0ll);
            s_col[tid] = (int)min(c0, (long long)a.cols);
        }
        s_start[tid] = block_scan(own, total, s_warp, TRIM_THREADS / 32) - own;
        __syncthreads();
        for (long long x = rank * TRIM_THREADS + tid; x < total; x += TRIM_CLUSTER * TRIM_THREADS) {
            int i = search_last(s_start, nr, x);
            int32_t* e = a.table + (int64_t)(r0 + i) * a.ld_table + s_col[i] + (x - s_start[i]);
            const int page = *e;
            *e = -1;
            if (page < 0 || page >= a.n_pages) continue;
            if (a.refs) {
                const int old = atomicSub(a.refs + page, 1);
                if (old <= 0) atomicAdd(a.refs + page, 1);
                if (old != 1) continue;
            }
            const int w = page >> 5;
            atom_or_cluster(map_to_cta(bits + (w % a.part) * 4, w / a.part), 1u << (page & 31));
        }
        __syncthreads();
    }
    cluster_sync_all();      // all bits are there
    long long mine = 0, total;
    for (int w = tid; w < a.part; w += TRIM_THREADS) mine += __popc(s_bits[w]);
    block_scan(mine, total, s_warp, TRIM_THREADS / 32);
    if (tid < TRIM_CLUSTER) st_cluster(map_to_cta(counts + rank * 4, tid), (uint32_t)total);
    __syncwarp();
    cluster_sync_all();
    int at = 0, all = 0;
    for (int b = 0; b < TRIM_CLUSTER; ++b) {
        if (b < rank) at += (int)s_count[b];
        all += (int)s_count[b];
    }
    if (rank == 0 && tid == 0) a.n_freed[0] = all;
    if (total == 0) return;
    for (int w0 = 0; w0 < a.part; w0 += TRIM_THREADS) {
        uint32_t b = w0 + tid < a.part ? s_bits[w0 + tid] : 0;
        const int c = __popc(b);
        long long chunk;
        int k = at + (int)block_scan(c, chunk, s_warp, TRIM_THREADS / 32) - c;
        for (; b; b &= b - 1) a.freed[k++] = (rank * a.part + w0 + tid) * 32 + __ffs((int)b) - 1;
        at += (int)chunk;
    }
}

cudaError_t launch_kv_trim(const KvTrimArgs& args, cudaStream_t st) {
    static PerDevice pd;
    KvTrimArgs a = args;
    a.part = std::max(1, (a.n_pages / 32 + 1 + TRIM_CLUSTER - 1) / TRIM_CLUSTER);
    cudaError_t e = opt_in_shared_memory(pd, kv_trim_kernel, TRIM_MAX_WORDS * 4);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(TRIM_CLUSTER);
    cfg.blockDim = dim3(TRIM_THREADS);
    cfg.dynamicSmemBytes = (size_t)a.part * 4;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = TRIM_CLUSTER;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kv_trim_kernel, a);
}

// ------------------------------------------------------------------------------------------------ kv_fork
// Row dst[i] of the table becomes a fork of row src[i], which holds `len` tokens: the full pages are shared (their counts of holders
// rise by one), and for tokens on a page that is not full the fork takes a page of its own from the free list, forks in order, and asks for a
// copy of those tokens.  (No row is both forked and a fork, so the lengths that block 0 writes are read by nobody.)  As in kv_slots every block scans the
// forks for itself; table entries are then shared out over the grid.  Latency: lengths -> scan -> search -> entry -> store, 5 to 6 us for 90 forks.
constexpr int FORK_THREADS = 256;

struct KvForkArgs {
    const int32_t* src;
    const int32_t* dst;
    int32_t* len;
    const int32_t* free_pages;
    int32_t* table;
    int64_t ld_table;
    int32_t* refs;           // may be null
    int32_t* copy_from;
    int32_t* copy_to;
    int32_t* copy_used;
    int32_t* taken;
    int n, R, page, n_free, cols, n_pages;
};

__global__ void __launch_bounds__(FORK_THREADS) kv_fork_kernel(const KvForkArgs a) {
    __shared__ long long s_start[FORK_THREADS], s_warp[32];
    __shared__ int s_src[FORK_THREADS], s_dst[FORK_THREADS];
    grid_launch_dependents();
    grid_dependency_wait();
    const int tid = threadIdx.x;
    long long carry = 0;      // pages taken by the forks before the chunk
    for (int i0 = 0; i0 < a.n; i0 += FORK_THREADS) {
        const int ni = min(FORK_THREADS, a.n - i0), i = i0 + tid;
        long long full = 0, need = 0, total, pages;
        int used = 0, src = -1, dst = -1, len = 0;
        if (tid < ni) {
            src = a.src[i];
            dst = a.dst[i];
            if (src >= 0 && src < a.R && dst >= 0 && dst < a.R && src != dst) {
                len = (int)min((long long)max(a.len[src], 0), (long long)a.cols * a.page);
                full = len / a.page;
                used = len % a.page;
                need = used > 0;
            } else {
                src = -1;
            }
            s_src[tid] = src;
            s_dst[tid] = dst;
        }
        s_start[tid] = block_scan(full, total, s_warp, FORK_THREADS / 32) - full;
        const long long first = carry + block_scan(need, pages, s_warp, FORK_THREADS / 32) - need;
        carry += pages;
        if (blockIdx.x == 0 && tid < ni) {
            int from = -1, to = -1, places = 0;
            if (need) {
                int page = first < a.n_free ? a.free_pages[first] : -1;
                if (page < 0 || page >= a.n_pages) page = -1;
                const int old = a.table[(int64_t)src * a.ld_table + full];
                a.table[(int64_t)dst * a.ld_table + full] = page;
                if (page >= 0 && a.refs) atomicAdd(a.refs + page, 1);
                if (page >= 0 && old >= 0 && old < a.n_pages) {
                    from = old;
                    to = page;
                    places = used;
                }
            }
            if (src >= 0) a.len[dst] = a.len[src];
            a.copy_from[i] = from;
            a.copy_to[i] = to;
            a.copy_used[i] = places;
        }
        __syncthreads();
        for (long long x = (long long)blockIdx.x * FORK_THREADS + tid; x < total; x += (long long)gridDim.x * FORK_THREADS) {
            const int k = search_last(s_start, ni, x);
            const int64_t col = x - s_start[k];
            const int page = a.table[(int64_t)s_src[k] * a.ld_table + col];
            a.table[(int64_t)s_dst[k] * a.ld_table + col] = page;
            if (a.refs && page >= 0 && page < a.n_pages) atomicAdd(a.refs + page, 1);
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) a.taken[0] = (int)carry;
}

cudaError_t launch_kv_fork(const KvForkArgs& a, int num_sms, cudaStream_t st) {
    const int64_t blocks = (int64_t)a.n * a.cols / (4 * FORK_THREADS) + 1;
    return launch_pdl(kv_fork_kernel, dim3((unsigned)std::min<int64_t>(blocks, num_sms)), dim3(FORK_THREADS), 0, st, a);
}

}  // namespace osc
