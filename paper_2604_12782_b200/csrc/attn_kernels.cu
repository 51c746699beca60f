// Attention of a step's new tokens over a paged key/value cache, in which groups of requests share a prefix.
//
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale * q . k_j,  lse = m + ln(sum_j exp(s_j - m))
//
// over all keys of the group's prefix and the own keys j <= kv_len - n + i of the request (i = index of the token
// among the request's n new ones).  The softmax is evaluated piecewise: any set of keys gives (m, l, O), two sets
// join as m = max, l = sum l_i 2^(m_i - m), O = sum O_i 2^(m_i - m) (everything in units of log2).
//
// The work is a list of segments: every group's prefix with the rows (tokens x query heads of one key/value head)
// of ALL its requests, then every request's own keys with its own rows.  So a prefix is read once per row tile, not
// once per request.  A segment is cut into units (row tile, key/value head), a unit into key tiles.  All key tiles
// of all units form one line that is cut into equal shares, one per CTA, whatever the lengths are: a CTA's share
// begins and ends inside a unit at most twice, so it leaves at most two pieces (m, l, O) in the workspace, joined
// by a last kernel.  The line is laid out by a one-CTA kernel from the lengths on the device; the host knows none.
//
// Segments with few rows run on the kernel of this file (16-row tiles, warp-level MMA: with 16 rows a key byte
// meets 16 multiply-adds, so HBM bounds it whatever the tensor path), segments with many rows on the
// tcgen05 kernel of the next file.
#include <cuda_bf16.h>

#include "common.cuh"

namespace osc {

constexpr int AT_FEW_ROWS = 16;              // rows of a few-row unit
constexpr int AT_FEW_KEYS = 64;              // keys of its tiles
constexpr int AT_WIDE_TILE = 128;            // rows of one tcgen05 tile; a wide unit has two of them
constexpr int AT_WIDE_KEYS = 128;
constexpr int AT_MAX_SMS = 148;
constexpr int AT_FEW_CTAS = 2 * AT_MAX_SMS;  // most CTAs of the few-row kernel (two per SM)
constexpr int AT_WIDE_CTAS = AT_MAX_SMS;

struct AttnPlan {            // filled by attn_plan_kernel
    int64_t* few_start;      // [S + 1] first tile of every segment on the few-row line
    int64_t* wide_start;     // [S + 1] ... on the tcgen05 line
    int32_t* req_group;      // [R] group of every request, -1: none (or a group whose prefix is empty)
};

struct AttnArgs {
    const uint16_t* q;
    int64_t ldq;
    uint16_t* o;
    int64_t ldo;
    float* lse;              // [T][Hq] or null
    const uint16_t* k;
    const uint16_t* v;
    int64_t page_stride, token_stride, head_stride;
    const int32_t* row_off;  // [R + 1]
    const int32_t* kv_len;   // [R]
    const int32_t* table;    // [R][ld_table]
    const int32_t* group_off;    // [P + 1]
    const int32_t* prefix_len;   // [P]
    const int32_t* ptable;       // [P][ld_ptable]
    int64_t ld_table, ld_ptable;
    int T, Hq, Hk, G, R, P, cols, pcols, page_shift, n_pages;
    int wide_min_rows;       // segments with at least this many rows per head go to the tcgen05 kernel
    int few_ctas, wide_ctas;
    float scale_log2;        // scale * log2(e)
    AttnPlan plan;
    float* dense[2];         // [T * Hq][D]: whole-unit results where a row has two sources (0: prefix, 1: own keys)
    float2* dense_ml[2];     // (m, l)
    float* few_part;         // [AT_FEW_CTAS][2][16][D]: first and last piece of every CTA
    float2* few_ml;
    float* wide_part;        // [AT_WIDE_CTAS][2][256][D]
    float2* wide_ml;
};

// ------------------------------------------------------------------------------------------------ segments
struct Segment {
    int t0, n;               // first row and number of tokens
    int klen;                // keys
    int causal;              // 1: own keys, token i sees klen - n + i + 1 of them; 0: prefix, every token sees klen
    const int32_t* pages;
    int npages;              // columns of the page list
};

// Lengths come from the device unchecked: rows are clamped to [0, T], keys to what the page list can name.
__device__ __forceinline__ int attn_row(const AttnArgs& a, int r) { return min(max(a.row_off[r], 0), a.T); }
__device__ __forceinline__ int attn_group(const AttnArgs& a, int g) { return min(max(a.group_off[g], 0), a.R); }
__device__ __forceinline__ int attn_keys(int len, int cols, int page_shift) {
    const int64_t room = (int64_t)cols << page_shift;
    return (int)min((int64_t)max(len, 0), min(room, (int64_t)0x40000000));
}
__device__ __forceinline__ Segment attn_segment(const AttnArgs& a, int s) {
    Segment g;
    int t1;
    if (s < a.P) {
        const int r0 = attn_group(a, s), r1 = max(attn_group(a, s + 1), r0);
        g.t0 = attn_row(a, r0);
        t1 = attn_row(a, r1);
        g.klen = attn_keys(a.prefix_len[s], a.pcols, a.page_shift);
        g.causal = 0;
        g.pages = a.ptable + (int64_t)s * a.ld_ptable;
        g.npages = a.pcols;
    } else {
        const int r = s - a.P;
        g.t0 = attn_row(a, r);
        t1 = attn_row(a, r + 1);
        g.klen = attn_keys(a.kv_len[r], a.cols, a.page_shift);
        g.causal = 1;
        g.pages = a.table + (int64_t)r * a.ld_table;
        g.npages = a.cols;
    }
    g.n = max(t1 - g.t0, 0);
    return g;
}
// keys that token i of the segment sees
__device__ __forceinline__ int seg_sees(const Segment& g, int i) { return g.causal ? max(g.klen - g.n + i + 1, 0) : g.klen; }
__device__ __forceinline__ bool seg_is_wide(const AttnArgs& a, const Segment& g) {
    return (int64_t)g.n * a.G >= a.wide_min_rows;
}

// The two kinds of units.  Few-row: 16 consecutive (token, head) rows.  Wide: two tiles of as many whole tokens as
// fit 128 rows.
struct FewUnits {
    static constexpr int KEYS = AT_FEW_KEYS;
    __device__ static int count(const AttnArgs& a, const Segment& g) { return (int)(((int64_t)g.n * a.G + AT_FEW_ROWS - 1) / AT_FEW_ROWS); }
    __device__ static int last_token(const AttnArgs& a, const Segment& g, int u) {
        return (int)min((int64_t)(g.n - 1), ((int64_t)u * AT_FEW_ROWS + AT_FEW_ROWS - 1) / a.G);
    }
    // own keys, all units but the last: ceil((klen - n + 1 + floor((16 u + 15) / G)) / 64)
    __device__ static void line(const AttnArgs& a, const Segment& g, int64_t& A, int64_t& B, int64_t& M, int64_t& u0) {
        const int64_t before = (int64_t)g.klen - g.n;
        A = AT_FEW_ROWS;
        B = a.G * (before + KEYS) + AT_FEW_ROWS - 1;
        M = (int64_t)KEYS * a.G;
        const int64_t need = -before * a.G - (AT_FEW_ROWS - 1);
        u0 = need > 0 ? (need + AT_FEW_ROWS - 1) / AT_FEW_ROWS : 0;
    }
};
struct WideUnits {
    static constexpr int KEYS = AT_WIDE_KEYS;
    __device__ static int tokens(const AttnArgs& a) { return 2 * (AT_WIDE_TILE / a.G); }
    __device__ static int count(const AttnArgs& a, const Segment& g) { return (int)(((int64_t)g.n + tokens(a) - 1) / tokens(a)); }
    __device__ static int last_token(const AttnArgs& a, const Segment& g, int u) {
        return (int)min((int64_t)g.n, ((int64_t)u + 1) * tokens(a)) - 1;
    }
    // own keys, all units but the last: ceil((klen - n + (u + 1) tokens) / 128)
    __device__ static void line(const AttnArgs& a, const Segment& g, int64_t& A, int64_t& B, int64_t& M, int64_t& u0) {
        const int64_t before = (int64_t)g.klen - g.n;
        A = tokens(a);
        B = before + A + KEYS - 1;
        M = KEYS;
        u0 = before < 0 ? -before / A : 0;
    }
};
template <class U>
__device__ __forceinline__ int unit_tiles(const AttnArgs& a, const Segment& g, int u) {
    return (seg_sees(g, U::last_token(a, g, u)) + U::KEYS - 1) / U::KEYS;
}
// sum over i < n of floor((a i + b) / m), for a, b >= 0 and m > 0, as in Euclid's algorithm
__device__ __forceinline__ int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
    int64_t sum = 0;
    while (n > 0) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const int64_t y = a * n + b;
        n = y / m;
        b = y % m;
        const int64_t t = m;
        m = a;
        a = t;
        if (n == 0) break;
    }
    return sum;
}
// key tiles of the units before unit u (u <= count) of one key/value head
template <class U>
__device__ __forceinline__ int64_t tiles_before(const AttnArgs& a, const Segment& g, int nu, int u) {
    if (u == 0 || g.klen == 0) return 0;
    if (!g.causal) return (int64_t)u * unit_tiles<U>(a, g, 0);
    int64_t sum = 0;
    if (u == nu) {                       // the last unit may be short
        sum = unit_tiles<U>(a, g, nu - 1);
        --u;
    }
    int64_t A, B, M, u0;
    U::line(a, g, A, B, M, u0);          // tiles(i) = floor((A i + B) / M) from unit u0 on, none before it
    if (u > u0) sum += floor_sum(u - u0, M, A, B + A * u0);
    return sum;
}
// key tiles of all units of one key/value head
template <class U>
__device__ __forceinline__ int64_t head_tiles(const AttnArgs& a, const Segment& g) {
    if (g.n == 0 || g.klen == 0) return 0;
    const int nu = U::count(a, g);
    return tiles_before<U>(a, g, nu, nu);
}

// Shares of the line of N tiles among C CTAs: CTA c has [floor(c N / C), floor((c + 1) N / C)).  Where the line is
// short, fewer CTAs share it, so that a share is at least MIN tiles: a piece costs its prologue and a join.
__device__ __forceinline__ int line_ctas(int64_t N, int ctas, int min_tiles) {
    const int64_t c = (N + min_tiles - 1) / min_tiles;
    return (int)(c < ctas ? (c < 1 ? 1 : c) : ctas);
}
__device__ __forceinline__ int64_t share_begin(int64_t N, int C, int c) { return N * c / C; }
// CTA whose share has tile x: the largest c with c N / C < x + 1
__device__ __forceinline__ int share_of(int64_t N, int C, int64_t x) { return (int)(((x + 1) * C - 1) / N); }
constexpr int AT_FEW_MIN_TILES = 1;
constexpr int AT_WIDE_MIN_TILES = 2;

// A position on a line: key tile kt of unit u of key/value head h of segment s.
template <class U>
struct Cursor {
    int s, h, u, kt, nu, nt;
    Segment g;
    __device__ void seek(const AttnArgs& a, const int64_t* start, int S, int64_t x) {
        int lo = 0, hi = S;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= x) lo = mid; else hi = mid;
        }
        s = lo;
        g = attn_segment(a, s);
        nu = U::count(a, g);
        const int64_t per_head = head_tiles<U>(a, g);
        int64_t y = x - start[s];
        h = (int)(y / per_head);
        y -= (int64_t)h * per_head;
        if (!g.causal) {
            nt = unit_tiles<U>(a, g, 0);
            u = (int)(y / nt);
            kt = (int)(y - (int64_t)u * nt);
        } else {
            int b = 0, e = nu;           // the last unit with at most y tiles before it
            while (e - b > 1) {
                const int mid = (b + e) >> 1;
                if (tiles_before<U>(a, g, nu, mid) <= y) b = mid; else e = mid;
            }
            u = b;
            nt = unit_tiles<U>(a, g, u);
            kt = (int)(y - tiles_before<U>(a, g, nu, u));
        }
    }
    // to the first tile of the next unit that has any; the caller knows that one exists
    __device__ void next_unit(const AttnArgs& a, const int64_t* start) {
        kt = 0;
        do {
            if (++u == nu) {
                u = 0;
                if (++h == a.Hk) {
                    h = 0;
                    do ++s; while (start[s + 1] == start[s]);
                    g = attn_segment(a, s);
                    nu = U::count(a, g);
                }
            }
            nt = unit_tiles<U>(a, g, u);
        } while (nt == 0);
    }
};

// first tile of unit u of head h of a segment
template <class U>
__device__ __forceinline__ int64_t unit_begin(const AttnArgs& a, const Segment& g, int64_t seg_start, int h, int u) {
    return seg_start + h * head_tiles<U>(a, g) + tiles_before<U>(a, g, U::count(a, g), u);
}

// ------------------------------------------------------------------------------------------------ the plan
constexpr int AT_PLAN_THREADS = 1024;

__global__ void __launch_bounds__(AT_PLAN_THREADS) attn_plan_kernel(const AttnArgs a) {
    __shared__ int64_t s_warp[2][AT_PLAN_THREADS / 32];
    grid_launch_dependents();
    grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, S = a.P + a.R;
    int64_t carry[2] = {0, 0};
    for (int s0 = 0; s0 < S; s0 += AT_PLAN_THREADS) {
        const int s = s0 + tid;
        int64_t own[2] = {0, 0}, inc[2];
        if (s < S) {
            const Segment g = attn_segment(a, s);
            if (seg_is_wide(a, g)) own[1] = head_tiles<WideUnits>(a, g) * a.Hk;
            else own[0] = head_tiles<FewUnits>(a, g) * a.Hk;
            if (s >= a.P) {
                int gr = -1;
                if (a.P > 0 && a.pcols > 0) {
                    int lo = 0, hi = a.P;          // the last group that begins at or before the request
                    while (hi - lo > 1) {
                        const int mid = (lo + hi) >> 1;
                        if (attn_group(a, mid) <= s - a.P) lo = mid; else hi = mid;
                    }
                    if (attn_group(a, lo) <= s - a.P && s - a.P < attn_group(a, lo + 1) && a.prefix_len[lo] > 0) gr = lo;
                }
                a.plan.req_group[s - a.P] = gr;
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            inc[j] = own[j];
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t up = __shfl_up_sync(0xFFFFFFFFu, inc[j], o);
                if (lane >= o) inc[j] += up;
            }
            if (lane == 31) s_warp[j][warp] = inc[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            int64_t before = carry[j], total = carry[j];
            for (int w = 0; w < AT_PLAN_THREADS / 32; ++w) {
                if (w < warp) before += s_warp[j][w];
                total += s_warp[j][w];
            }
            if (s < S) (j ? a.plan.wide_start : a.plan.few_start)[s] = before + inc[j] - own[j];
            carry[j] = total;
        }
        __syncthreads();
    }
    if (tid == 0) {
        a.plan.few_start[S] = carry[0];
        a.plan.wide_start[S] = carry[1];
    }
}

// --------------------------------------------------------------------------------------------- few rows
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The running maximum that P and l are taken against moves only when a score passes it by more than 2^8: the
// quotient O / l does not depend on it, and 2^8 more in every term costs no bit of fp32 or bf16.
constexpr float AT_SLACK = 8.0f;
constexpr int AT_FEW_THREADS = 128;

template <int D>
struct FewCfg {
    static constexpr int KV_BYTES = 16 * D * 2;                  // one warp's 16 keys (or values) of a tile
    static constexpr int SLOT_BYTES = 2 * KV_BYTES;
    static constexpr int STAGES = D == 128 ? 3 : 6;
    static constexpr int RING = 4 * STAGES * SLOT_BYTES;         // every warp has its own ring
    static constexpr int JOIN = 2 * (16 * D * 4 + 16 * 8);       // two warps' (O, m, l) on the way to two others
    static constexpr int SMEM = RING + JOIN;
};

// One CTA: four warps, each on its own 16 keys of every 64-key tile with its own ring of cp.async slots and its own
// (m, l, O), so that no barrier runs inside the key loop; the four results are joined through shared memory at the
// end of a unit.  The loads run on over the ends of units.  A page number is fetched one tile ahead of the
// loads that need it.
template <int D>
__global__ void __launch_bounds__(AT_FEW_THREADS, 2) attn_few_kernel(const AttnArgs a) {
    using C = FewCfg<D>;
    constexpr int NJ = D / 8;          // 8-channel column blocks of O
    constexpr int KS = D / 16;         // k steps of Q K^T
    constexpr int CHUNKS = D / 8;      // 16-byte chunks of a key
    extern __shared__ __align__(128) uint8_t at_smem[];
    grid_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    const int S = a.P + a.R;
    const int64_t N = a.plan.few_start[S];
    if (N == 0) return;
    const int nc = line_ctas(N, a.few_ctas, AT_FEW_MIN_TILES);
    if ((int)blockIdx.x >= nc) return;
    const int64_t x0 = share_begin(N, nc, blockIdx.x), x1 = share_begin(N, nc, blockIdx.x + 1);
    if (x0 >= x1) return;

    const uint32_t ring = smem_u32(at_smem) + warp * C::STAGES * C::SLOT_BYTES;
    float* join = reinterpret_cast<float*>(at_smem + C::RING);

    Cursor<FewUnits> cur, ld;
    cur.seek(a, a.plan.few_start, S, x0);
    ld = cur;
    const int page_mask = (1 << a.page_shift) - 1;
    const int kw = warp * 16;          // first key of the warp inside a tile
    // page that holds the warp's 16 keys of the loader's tile (a page has at least 16 tokens)
    auto page_of = [&]() -> int {
        const int key = ld.kt * AT_FEW_KEYS + kw;
        if (key >= ld.g.klen) return -1;
        const int c = key >> a.page_shift;
        const int p = c < ld.g.npages ? ld.g.pages[c] : -1;
        return (p >= 0 && p < a.n_pages) ? p : -1;
    };
    int64_t xl = x0;                   // loader's position
    int page = page_of();
    auto load = [&](int slot) {
        if (xl < x1) {
            const int key = ld.kt * AT_FEW_KEYS + kw;
            const int64_t base = (int64_t)max(page, 0) * a.page_stride + (int64_t)(key & page_mask) * a.token_stride + (int64_t)ld.h * a.head_stride;
            const uint32_t dst = ring + slot * C::SLOT_BYTES;
            const int nvalid = page >= 0 ? ld.g.klen - key : 0;   // keys past the end (and absent pages) read as zero
#pragma unroll
            for (int i = 0; i < 16 * CHUNKS / 32; ++i) {
                const int r = (i * 32 + lane) / CHUNKS, c = (i * 32 + lane) % CHUNKS;
                const int64_t off = r < nvalid ? base + (int64_t)r * a.token_stride + c * 8 : 0;
                const uint32_t d = dst + r * (D * 2) + ((c ^ (r & 7)) * 16);
                cp_async_16(d, a.k + off, r < nvalid);
                cp_async_16(d + C::KV_BYTES, a.v + off, r < nvalid);
            }
            if (++xl < x1) {
                if (++ld.kt == ld.nt) ld.next_unit(a, a.plan.few_start);
                page = page_of();
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) load(i);

    const int r0 = lane >> 2, cq = lane & 3;       // the thread's rows r0, r0 + 8 and column pair of an MMA fragment
    int slot = 0, fill = C::STAGES - 1;
    int64_t x = x0;
    while (x < x1) {
        // ---- a unit (or the share's part of it)
        const int row0 = cur.u * AT_FEW_ROWS;
        const int nrows = (int)min((int64_t)AT_FEW_ROWS, (int64_t)cur.g.n * a.G - row0);
        uint32_t qf[KS][4];
        int sees[2];
#pragma unroll
        for (int hlf = 0; hlf < 2; ++hlf) {
            const int r = r0 + hlf * 8;
            const int tok = (row0 + r) / a.G, hd = (row0 + r) % a.G;
            const bool ok = r < nrows;
            sees[hlf] = ok ? seg_sees(cur.g, tok) : 0;
            const uint16_t* qp = a.q + (ok ? (int64_t)(cur.g.t0 + tok) * a.ldq + (int64_t)(cur.h * a.G + hd) * D : 0) + cq * 2;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[ks][hlf] = ok ? *reinterpret_cast<const uint32_t*>(qp + ks * 16) : 0u;
                qf[ks][hlf + 2] = ok ? *reinterpret_cast<const uint32_t*>(qp + ks * 16 + 8) : 0u;
            }
        }
        float o[NJ][4];
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
        const int64_t unit_x0 = x - cur.kt, unit_x1 = unit_x0 + cur.nt;
        const int64_t xe = min(unit_x1, x1);
        for (; x < xe; ++x, ++cur.kt) {
            load(fill);
            if (++fill == C::STAGES) fill = 0;
            cp_async_wait<C::STAGES - 1>();
            __syncwarp();
            const uint32_t kb = ring + slot * C::SLOT_BYTES, vb = kb + C::KV_BYTES;
            const int key0 = cur.kt * AT_FEW_KEYS + kw;
            if (key0 < cur.g.klen) {
                float sc[2][4] = {};
                {
                    const int r = (lane & 7) + ((lane >> 4) << 3), ch = (lane >> 3) & 1;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        uint32_t b[4];
                        ldsm_x4(kb + r * (D * 2) + (((ks * 2 + ch) ^ (r & 7)) * 16), b);
                        mma_16816(sc[0], qf[ks], b[0], b[1]);
                        mma_16816(sc[1], qf[ks], b[2], b[3]);
                    }
                }
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + n8 * 8 + cq * 2 + (e & 1);
                        sc[n8][e] = key < sees[e >> 1] ? sc[n8][e] * a.scale_log2 : -INFINITY;
                        mx[e >> 1] = fmaxf(mx[e >> 1], sc[n8][e]);
                    }
                bool move = false;
#pragma unroll
                for (int hlf = 0; hlf < 2; ++hlf) {
                    mx[hlf] = fmaxf(mx[hlf], __shfl_xor_sync(0xFFFFFFFFu, mx[hlf], 1));
                    mx[hlf] = fmaxf(mx[hlf], __shfl_xor_sync(0xFFFFFFFFu, mx[hlf], 2));
                    move |= mx[hlf] > m[hlf] + AT_SLACK;
                }
                if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
                    for (int hlf = 0; hlf < 2; ++hlf) {
                        const float mn = fmaxf(m[hlf], mx[hlf]);
                        const float f = mn == -INFINITY ? 1.0f : exp2_approx(m[hlf] - mn);
                        m[hlf] = mn;
                        l[hlf] *= f;
#pragma unroll
                        for (int j = 0; j < NJ; ++j) { o[j][2 * hlf] *= f; o[j][2 * hlf + 1] *= f; }
                    }
                }
                uint32_t pf[4];
                float p[2][4];
#pragma unroll
                for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ref = m[e >> 1] == -INFINITY ? 0.0f : m[e >> 1];
                        p[n8][e] = exp2_approx(sc[n8][e] - ref);
                        l[e >> 1] += p[n8][e];
                    }
#pragma unroll
                for (int n8 = 0; n8 < 2; ++n8) {
                    pf[2 * n8] = bf162_bits(__floats2bfloat162_rn(p[n8][0], p[n8][1]));
                    pf[2 * n8 + 1] = bf162_bits(__floats2bfloat162_rn(p[n8][2], p[n8][3]));
                }
                const int r = lane & 15, ch = lane >> 4;
#pragma unroll
                for (int j = 0; j < NJ; j += 2) {
                    uint32_t b[4];
                    ldsm_x4_trans(vb + r * (D * 2) + (((j + ch) ^ (r & 7)) * 16), b);
                    mma_16816(o[j], pf, b[0], b[1]);
                    mma_16816(o[j + 1], pf, b[2], b[3]);
                }
            }
            __syncwarp();              // the slot is filled again by the next load
            if (++slot == C::STAGES) slot = 0;
        }
        // ---- join the four warps: 2, 3 -> 0, 1, then 1 -> 0
#pragma unroll
        for (int hlf = 0; hlf < 2; ++hlf) {
            l[hlf] += __shfl_xor_sync(0xFFFFFFFFu, l[hlf], 1);
            l[hlf] += __shfl_xor_sync(0xFFFFFFFFu, l[hlf], 2);
        }
#pragma unroll
        for (int step = 2; step >= 1; step >>= 1) {
            if (warp >= step && warp < 2 * step) {
                float* buf = join + (warp - step) * (16 * D + 32);
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    *reinterpret_cast<float2*>(buf + r0 * D + j * 8 + cq * 2) = make_float2(o[j][0], o[j][1]);
                    *reinterpret_cast<float2*>(buf + (r0 + 8) * D + j * 8 + cq * 2) = make_float2(o[j][2], o[j][3]);
                }
                if (cq == 0) {
                    *reinterpret_cast<float2*>(buf + 16 * D + r0 * 2) = make_float2(m[0], l[0]);
                    *reinterpret_cast<float2*>(buf + 16 * D + (r0 + 8) * 2) = make_float2(m[1], l[1]);
                }
            }
            __syncthreads();
            if (warp < step) {
                const float* buf = join + warp * (16 * D + 32);
#pragma unroll
                for (int hlf = 0; hlf < 2; ++hlf) {
                    const int r = r0 + hlf * 8;
                    const float2 ml = *reinterpret_cast<const float2*>(buf + 16 * D + r * 2);
                    const float mn = fmaxf(m[hlf], ml.x);
                    const float f0 = mn == -INFINITY ? 0.0f : exp2_approx(m[hlf] - mn), f1 = mn == -INFINITY ? 0.0f : exp2_approx(ml.x - mn);
                    m[hlf] = mn;
                    l[hlf] = l[hlf] * f0 + ml.y * f1;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const float2 v = *reinterpret_cast<const float2*>(buf + r * D + j * 8 + cq * 2);
                        o[j][2 * hlf] = o[j][2 * hlf] * f0 + v.x * f1;
                        o[j][2 * hlf + 1] = o[j][2 * hlf + 1] * f0 + v.y * f1;
                    }
                }
            }
            __syncthreads();
        }
        if (warp == 0) {
            const bool split = unit_x0 < x0 || unit_x1 > x1;
            const bool two = cur.s < a.P || a.plan.req_group[cur.s - a.P] >= 0;   // the rows have (or may have) another source
#pragma unroll
            for (int hlf = 0; hlf < 2; ++hlf) {
                const int r = r0 + hlf * 8;
                if (r >= nrows) continue;
                const int64_t row = (int64_t)(cur.g.t0 + (row0 + r) / a.G) * a.Hq + cur.h * a.G + (row0 + r) % a.G;
                if (!split && !two) {
                    const float inv = l[hlf] > 0.0f || l[hlf] != l[hlf] ? 1.0f / l[hlf] : 0.0f;
                    uint16_t* op = a.o + (int64_t)(row / a.Hq) * a.ldo + (row % a.Hq) * D + cq * 2;
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        *reinterpret_cast<uint32_t*>(op + j * 8) = bf162_bits(__floats2bfloat162_rn(o[j][2 * hlf] * inv, o[j][2 * hlf + 1] * inv));
                    if (a.lse && cq == 0) a.lse[row] = l[hlf] == 0.0f ? -INFINITY : (m[hlf] + log2f(l[hlf])) * 0.69314718055994531f;
                } else {
                    const int64_t at = split ? ((int64_t)blockIdx.x * 2 + (unit_x0 > x0 ? 1 : 0)) * AT_FEW_ROWS + r : row;
                    float* part = split ? a.few_part : a.dense[cur.s >= a.P];
                    float2* ml = split ? a.few_ml : a.dense_ml[cur.s >= a.P];
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        *reinterpret_cast<float2*>(part + at * D + j * 8 + cq * 2) = make_float2(o[j][2 * hlf], o[j][2 * hlf + 1]);
                    if (cq == 0) ml[at] = make_float2(m[hlf], l[hlf]);
                }
            }
        }
        if (x < x1) cur.next_unit(a, a.plan.few_start);
    }
    cp_async_wait<0>();
}

// ------------------------------------------------------------------------------------------------- join
// One CTA per (token, key/value head): finds the token's request, walks over the pieces of its rows in the order of
// the line (so the result does not depend on which CTA was first) and writes o and lse.  Rows that a unit wrote
// itself (all their keys in one unit) are left alone; rows without any key become 0 and -inf.
constexpr int AT_JOIN_THREADS = 128;

// Adds the pieces of one row from one segment.  `which` 0: prefix, 1: own keys.
template <int D, class U, class F>
__device__ __forceinline__ void join_pieces(const AttnArgs& a, const Segment& g, int64_t N, int ctas, int min_tiles, int64_t seg_start,
                                            int h, int u, int row_in_unit, int unit_rows, const float* part, const float2* ml,
                                            const float* dense, const float2* dense_ml, int64_t dense_row, F add) {
    const int nt = unit_tiles<U>(a, g, u);
    if (nt == 0) return;
    const int C = line_ctas(N, ctas, min_tiles);
    const int64_t b = unit_begin<U>(a, g, seg_start, h, u), e = b + nt;
    const int c0 = share_of(N, C, b), c1 = share_of(N, C, e - 1);
    if (c0 == c1) { add(dense + dense_row * D, dense_ml[dense_row]); return; }
    for (int c = c0; c <= c1; ++c) {
        const int64_t at = ((int64_t)c * 2 + (b > share_begin(N, C, c) ? 1 : 0)) * unit_rows + row_in_unit;
        add(part + at * D, ml[at]);
    }
}

template <int D>
__global__ void __launch_bounds__(AT_JOIN_THREADS) attn_join_kernel(const AttnArgs a) {
    constexpr int V = D / 32;          // channels per lane
    __shared__ int s_req;
    grid_launch_dependents();
    grid_dependency_wait();
    const int t = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) s_req = -1;
    __syncthreads();
    for (int r = tid; r < a.R; r += AT_JOIN_THREADS)
        if (attn_row(a, r) <= t && t < attn_row(a, r + 1)) s_req = r;
    __syncthreads();
    const int r = s_req;
    if (r < 0) return;                 // behind the last request: left as it is
    const int S = a.P + a.R;
    const int grp = a.plan.req_group[r];
    const int64_t nf = a.plan.few_start[S], nw = a.plan.wide_start[S];
    const Segment own = attn_segment(a, a.P + r);
    Segment pre = own;
    if (grp >= 0) pre = attn_segment(a, grp);
    for (int g = warp; g < a.G; g += AT_JOIN_THREADS / 32) {
        const int hq = h * a.G + g;
        const int64_t row = (int64_t)t * a.Hq + hq;
        float m = -INFINITY, l = 0.0f, o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = 0.0f;
        auto add = [&](const float* part, float2 ml) {
            const float mn = fmaxf(m, ml.x);
            if (mn == -INFINITY) return;
            const float f0 = exp2_approx(m - mn), f1 = exp2_approx(ml.x - mn);
            m = mn;
            l = l * f0 + ml.y * f1;
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = o[j] * f0 + part[lane * V + j] * f1;
        };
        bool direct = false;
        for (int which = grp >= 0 ? 0 : 1; which < 2; ++which) {
            const Segment& sg = which ? own : pre;
            const int s = which ? a.P + r : grp;
            const int tok = t - sg.t0;
            if (sg.klen == 0 || tok < 0 || tok >= sg.n) continue;
            if (seg_is_wide(a, sg)) {
                const int tpt = AT_WIDE_TILE / a.G, u = tok / (2 * tpt), in = tok % (2 * tpt);
                if (which && grp < 0) {
                    const int nt = unit_tiles<WideUnits>(a, sg, u);
                    const int C = line_ctas(nw, a.wide_ctas, AT_WIDE_MIN_TILES);
                    const int64_t b = nt ? unit_begin<WideUnits>(a, sg, a.plan.wide_start[s], h, u) : 0;
                    if (nt && share_of(nw, C, b) == share_of(nw, C, b + nt - 1)) { direct = true; continue; }
                }
                const int rin = (in / tpt) * AT_WIDE_TILE + (in % tpt) * a.G + g;
                join_pieces<D, WideUnits>(a, sg, nw, a.wide_ctas, AT_WIDE_MIN_TILES, a.plan.wide_start[s], h, u, rin, 2 * AT_WIDE_TILE,
                                          a.wide_part, a.wide_ml, a.dense[which], a.dense_ml[which], row, add);
            } else {
                const int fr = tok * a.G + g, u = fr / AT_FEW_ROWS;
                if (which && grp < 0) {
                    const int nt = unit_tiles<FewUnits>(a, sg, u);
                    const int C = line_ctas(nf, a.few_ctas, AT_FEW_MIN_TILES);
                    const int64_t b = nt ? unit_begin<FewUnits>(a, sg, a.plan.few_start[s], h, u) : 0;
                    if (nt && share_of(nf, C, b) == share_of(nf, C, b + nt - 1)) { direct = true; continue; }
                }
                join_pieces<D, FewUnits>(a, sg, nf, a.few_ctas, AT_FEW_MIN_TILES, a.plan.few_start[s], h, u, fr % AT_FEW_ROWS, AT_FEW_ROWS,
                                         a.few_part, a.few_ml, a.dense[which], a.dense_ml[which], row, add);
            }
        }
        if (direct) continue;
        const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
        uint16_t* op = a.o + (int64_t)t * a.ldo + (int64_t)hq * D + lane * V;
        if (V == 4) {
            *reinterpret_cast<uint2*>(op) = make_uint2(bf162_bits(__floats2bfloat162_rn(o[0] * inv, o[1] * inv)),
                                                       bf162_bits(__floats2bfloat162_rn(o[V - 2] * inv, o[V - 1] * inv)));
        } else {
            *reinterpret_cast<uint32_t*>(op) = bf162_bits(__floats2bfloat162_rn(o[0] * inv, o[1] * inv));
        }
        if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
    }
}

}  // namespace osc
