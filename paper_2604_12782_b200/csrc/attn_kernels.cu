// Attention of a step's new tokens over a paged key/value cache, in which groups of requests share a prefix.
//
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale * q . k_j,  lse = m + ln(sum_j exp(s_j - m))
//
// over all keys of the group's prefix and the own keys j <= kv_len - n + i of the request (i = index of the token
// among the request's n new ones).  With a mask (trees of drafted tokens) a row sees all own keys before the new tokens, and
// of those the ones whose bits are set in its row of the mask.  The softmax is evaluated piecewise: any set of keys gives (m, l, O), two sets
// join as m = max, l = sum l_i 2^(m_i - m), O = sum O_i 2^(m_i - m) (everything in units of log2).
//
// The work is a list of segments: every group's prefix with the rows (tokens x query heads of one key/value head)
// of ALL its requests, then every request's own keys with its own rows.  So a prefix is read once per row tile, not
// once per request.  Where every request of a group fills row tiles by itself (prompts), nothing is gained by
// packing their rows together, and a request's keys are one list instead: prefix, then own keys.
// A segment is cut into units (row tile, key/value heads), a unit into key tiles.  All key tiles of all units form
// one line that is cut into equal shares, one per CTA, whatever the lengths are: a CTA's share begins and ends
// inside a unit at most twice, so it leaves at most two pieces (m, l, O) in the workspace, joined by a last
// kernel.  The line is laid out by a one-CTA kernel from the lengths on the device; the host knows none.
//
// Segments with few rows run on the kernel of this file (16-row tiles, warp-level MMA: with 16 rows a key byte
// meets 16 multiply-adds, so HBM bounds it whatever the tensor path), segments with many rows on the
// tcgen05 kernel of the next file.
#include <cuda_bf16.h>

#include "common.cuh"

namespace osc {

constexpr int AT_FEW_ROWS = 16;              // rows of a few-row unit
constexpr int AT_WIDE_TILE = 128;            // rows of one tcgen05 tile; a wide unit has two of them
constexpr int AT_WIDE_KEYS = 128;            // keys of its tiles
constexpr int AT_MERGE_ROWS = 2 * AT_WIDE_TILE;  // a group whose requests all have at least this many rows has no prefix segment
constexpr int AT_MAX_SMS = 148;
constexpr int AT_FEW_CTAS = 4 * AT_MAX_SMS;  // most CTAs of the few-row kernel (two per SM at a time)
constexpr int AT_FEW_HEADS = 4;              // most key/value heads of a few-row unit
constexpr int AT_WIDE_CTAS = AT_MAX_SMS;

// A segment as the plan leaves it in the workspace (two 16-byte loads).
struct __align__(16) Segment {
    int t0, n;               // first row and number of tokens
    int klen;                // keys: the prefix, or the request's own
    int plen;                // keys of the group's prefix in front of the own keys (merged groups), else 0
    int tiles;               // places of all units of one head (of one head group on the few-row line): key tiles, and LEAD a unit
    int start;               // its first place on its line
    int group;               // of a request: its group, -1: none (or one with an empty prefix)
    int flags;
};
constexpr int SEG_WIDE = 1;  // on the tcgen05 line
constexpr int SEG_OWN = 4;   // own keys without a mask: token i sees klen - n + i + 1 of them; else every token meets all klen (a prefix, or masked)
constexpr int SEG_TWO = 2;   // the rows have another source: O goes to the workspace, and the join looks at every row

// A unit that the end of a CTA's share cuts, told by the first CTA that meets it; the join finds its pieces by it.
struct __align__(16) CutUnit {
    int begin, share;        // (last) place of its first tile, and the places of a share
    int tiles;               // 0: the share ends with a unit, or the unit's rows have two sources, or it was cut before
    int h, u;                // head (group) and row unit
    int t0, n;               // rows of the segment
    int weight;              // places of a tile
};

struct AttnPlan {            // filled by attn_plan_kernel
    int32_t* few_start;      // [S + 1] first tile of every segment on the few-row line
    int32_t* wide_start;     // [S + 1] ... on the tcgen05 line
    Segment* seg;            // [S]
    int32_t* tok_req;        // [T], where there are prefixes: the request of every token whose rows have two sources, else -1;
                             // not written where no request covers the token
    int32_t* share;          // [3]: tiles of a share on the few-row line, on the tcgen05 line; whether any row has two sources
    CutUnit* cut[2];         // [AT_FEW_CTAS], [AT_WIDE_CTAS]: filled by the attention kernels
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
    int T, Hq, Hk, G, head_dim, R, P, cols, pcols, page_shift, n_pages;
    int wide_min_rows;       // segments with at least this many rows per head go to the tcgen05 kernel
    int inv_g;               // ceil(2^16 / G): x / G = x * inv_g >> 16 for x < 128
    int tpt;                 // whole tokens that fit the 128 rows of a tcgen05 tile
    int few_hw;              // heads of a few-row unit: 4, 2 or 1
    int few_ctas, wide_ctas;
    int self;                // no plan kernel in front of the tcgen05 kernel (masked calls only)
    float scale_log2;        // scale * log2(e)
    const uint32_t* mask;    // [T][ld_mask], null: tokens see the new tokens before them.  Bit m % 32 of word m / 32: the row sees new token m
    int64_t ld_mask;
    int words;               // of a row of the mask
    AttnPlan plan;
    // Partial results, row by row: O [D] in part, (m, l) in ml.  Rows [0, AT_FEW_SLOTS): the first and the last piece of every few-row
    // CTA ([CTA][2][few_hw][16]); then those of the tcgen05 CTAs ([CTA][2][256]); then, where there are prefixes, twice T * Hq rows
    // for whole units of rows with two sources (prefix, own keys).
    float* part;
    float2* ml;
};
constexpr int AT_FEW_SLOTS = AT_FEW_CTAS * 2 * AT_FEW_HEADS * AT_FEW_ROWS;
constexpr int AT_WIDE_SLOTS = AT_WIDE_CTAS * 2 * 2 * AT_WIDE_TILE;
__device__ __forceinline__ int dense_row(const AttnArgs& a, int own, int row) { return AT_FEW_SLOTS + AT_WIDE_SLOTS + own * a.T * a.Hq + row; }

// ------------------------------------------------------------------------------------------------ segments
// What the plan wrote is read past L1: the few-row kernel may begin before the kernel behind the plan has ended.
__device__ __forceinline__ int load_plan(const int32_t* p) { return __ldcg(p); }

// Lengths come from the device unchecked: rows are clamped to [0, T], keys to what the page list can name.
__device__ __forceinline__ int attn_row(const AttnArgs& a, int r) { return min(max(a.row_off[r], 0), a.T); }
__device__ __forceinline__ int attn_group(const AttnArgs& a, int g) { return min(max(a.group_off[g], 0), a.R); }
__device__ __forceinline__ int attn_keys(int len, int cols, int page_shift) {
    const int64_t room = (int64_t)cols << page_shift;
    return (int)min((int64_t)max(len, 0), min(room, (int64_t)0x20000000));
}
// page list of the segment's own keys, and of the prefix in front of them
__device__ __forceinline__ const int32_t* seg_pages(const AttnArgs& a, int s) {
    return s < a.P ? a.ptable + (int64_t)s * a.ld_ptable : a.table + (int64_t)(s - a.P) * a.ld_table;
}
// keys that token i of the segment sees, without the prefix in front
__device__ __forceinline__ int seg_sees(const Segment& g, int i) { return g.flags & SEG_OWN ? max(g.klen - g.n + i + 1, 0) : g.klen; }

// tokens of a request, its first ones, that see no own key, as far as lengths tell
__device__ __forceinline__ int seg_blind(const AttnArgs& a, const Segment& g) { return a.mask ? (g.klen > 0 ? 0 : g.n) : max(g.n - g.klen, 0); }

// Which of the 32 own keys from `key` on a row with the given mask row sees: those before the first new token (at ctx, which is
// negative where the cache holds less than all new tokens), then by the mask's bits, none from klen on.  Words past the row's last read as 0.
__device__ __forceinline__ uint32_t mask_word(const AttnArgs& a, const uint32_t* row, int w) { return (unsigned)w < (unsigned)a.words ? row[w] : 0u; }
__device__ __forceinline__ uint32_t tree_sees(const AttnArgs& a, const uint32_t* row, int key, int ctx, int klen) {
    const int m = key - ctx;
    uint32_t bits = 0xFFFFFFFFu;
    if (m > -32) {
        const int w = m >> 5;            // -1 where the 32 keys begin before the first new token
        bits = __funnelshift_r(w < 0 ? 0xFFFFFFFFu : mask_word(a, row, w), mask_word(a, row, w + 1), m & 31);
    }
    const int left = klen - key;
    return left >= 32 ? bits : left > 0 ? bits & ((1u << left) - 1u) : 0u;
}

// bf16 pairs: whether one of the two is an Inf or a NaN, and the pair with those replaced by 0
__device__ __forceinline__ bool has_odd(uint32_t x) { return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u; }
__device__ __forceinline__ bool has_odd(const uint4& x) { return has_odd(x.x) || has_odd(x.y) || has_odd(x.z) || has_odd(x.w); }
__device__ __forceinline__ uint32_t drop_odd(uint32_t x) {
    if ((x & 0x7F80u) == 0x7F80u) x &= 0xFFFF0000u;
    return (x & 0x7F800000u) == 0x7F800000u ? x & 0xFFFFu : x;
}
__device__ __forceinline__ uint4 drop_odd(const uint4& x) { return make_uint4(drop_odd(x.x), drop_odd(x.y), drop_odd(x.z), drop_odd(x.w)); }

// Rows of a segment (tokens x heads of one key/value head) and of all segments are ints: the host has seen to T * n_q <= 2^29.
// The two kinds of units.  Few-row: 16 consecutive (token, head) rows of one token list, few_hw heads side by side, tiles
// of 64 / few_hw keys.  Wide: two tiles of as many whole tokens as fit 128 rows, one head.
struct FewUnits {
    static constexpr int LEAD = 0;     // tiles' places on the line in front of a unit's tiles
    __device__ static int weight(const AttnArgs&, const Segment&, int) { return 1; }     // places of a tile
    __device__ static int key_shift(const AttnArgs& a) { return a.few_hw == 4 ? 4 : a.few_hw == 2 ? 5 : 6; }
    __device__ static int heads(const AttnArgs& a) { return a.Hk / a.few_hw; }
    __device__ static int count(const AttnArgs& a, const Segment& g) { return (g.n * a.G + AT_FEW_ROWS - 1) / AT_FEW_ROWS; }
    __device__ static int last_token(const AttnArgs& a, const Segment& g, int u) {
        return min(g.n - 1, (u * AT_FEW_ROWS + AT_FEW_ROWS - 1) / a.G);
    }
    // own keys, all units but the last: ceil((klen - n + 1 + floor((16 u + 15) / G)) / KEYS)
    __device__ static void line(const AttnArgs& a, const Segment& g, int64_t& A, int64_t& B, int64_t& M, int64_t& u0) {
        const int64_t before = (int64_t)g.klen - g.n, keys = 1 << key_shift(a);
        A = AT_FEW_ROWS;
        B = a.G * (before + keys) + AT_FEW_ROWS - 1;
        M = keys * a.G;
        const int64_t need = -before * a.G - (AT_FEW_ROWS - 1);
        u0 = need > 0 ? (need + AT_FEW_ROWS - 1) / AT_FEW_ROWS : 0;
    }
};
struct WideUnits {
    static constexpr int LEAD = 4;     // a unit costs about that many tiles beside its own: Q, an empty and a filling pipeline, O
    // Requests with a tree each are units with one row tile or with two, in any mixture.  A key tile takes 1.1 to 1.25 us with one and 1.6 to 1.7 with two
    // (five requests of 40000 keys, and 24 of 4200, HBM saturated): two places to three.  With the same place for all the CTAs of the five requests ended between
    // 147 and 227 us.  Prompts without a mask fill both row tiles nearly always.
    __device__ static int weight(const AttnArgs& a, const Segment& g, int u) { return !a.mask ? 1 : g.n - u * tokens(a) > a.tpt ? 3 : 2; }
    __device__ static constexpr int key_shift(const AttnArgs&) { return 7; }
    __device__ static int heads(const AttnArgs& a) { return a.Hk; }
    __device__ static int tokens(const AttnArgs& a) { return 2 * a.tpt; }
    __device__ static int count(const AttnArgs& a, const Segment& g) { return (g.n + tokens(a) - 1) / tokens(a); }
    __device__ static int last_token(const AttnArgs& a, const Segment& g, int u) {
        return min(g.n, (u + 1) * tokens(a)) - 1;
    }
    // own keys, all units but the last: ceil((klen - n + (u + 1) tokens) / 128)
    __device__ static void line(const AttnArgs& a, const Segment& g, int64_t& A, int64_t& B, int64_t& M, int64_t& u0) {
        const int64_t before = (int64_t)g.klen - g.n;
        A = tokens(a);
        B = before + A + AT_WIDE_KEYS - 1;
        M = AT_WIDE_KEYS;
        u0 = before < 0 ? -before / A : 0;
    }
};
// tiles of the prefix in front, and of the whole unit
template <class U>
__device__ __forceinline__ int front_tiles(const AttnArgs& a, const Segment& g) {
    return (g.plen + (1 << U::key_shift(a)) - 1) >> U::key_shift(a);
}
template <class U>
__device__ __forceinline__ int unit_tiles(const AttnArgs& a, const Segment& g, int u) {
    return front_tiles<U>(a, g) + ((seg_sees(g, U::last_token(a, g, u)) + (1 << U::key_shift(a)) - 1) >> U::key_shift(a));
}
template <class U>
__device__ __forceinline__ int unit_span(int tiles, int weight) { return tiles ? (tiles + U::LEAD) * weight : 0; }
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
constexpr int AT_LOOP_UNITS = 64;
// places on the line of the units before unit u (u <= count) of one head; the host has seen to it that they are ints
template <class U>
__device__ __forceinline__ int span_before(const AttnArgs& a, const Segment& g, int nu, int u) {
    if (u == 0) return 0;
    if (!(g.flags & SEG_OWN)) {              // all units but the last have the same weight
        const int tiles = unit_tiles<U>(a, g, 0), all = u == nu ? 1 : 0;
        return (u - all) * unit_span<U>(tiles, U::weight(a, g, 0)) + all * unit_span<U>(tiles, U::weight(a, g, nu - 1));
    }
    const int front = front_tiles<U>(a, g);
    int sum = u * front, some = front ? u : 0;   // tiles, and units that have any
    if (g.klen > 0) {
        if (u == nu) {                   // the last unit may be short
            --u;
            const int last = (seg_sees(g, U::last_token(a, g, u)) + (1 << U::key_shift(a)) - 1) >> U::key_shift(a);
            sum += last;
            if (!front && last) ++some;
        }
        int64_t A, B, M, u0;
        U::line(a, g, A, B, M, u0);      // own tiles(i) = floor((A i + B) / M) >= 1 from unit u0 on, none before it
        if (u > u0) {
            if (!front) some += (int)(u - u0);
            if (u - u0 <= AT_LOOP_UNITS) {   // nearly always: a short loop, where the closed form's 64-bit divisions take longer
#pragma unroll 1
                for (int i = (int)u0; i < u; ++i) sum += unit_tiles<U>(a, g, i) - front;
            } else {
                sum += (int)floor_sum(u - u0, M, A, B + A * u0);
            }
        }
    }
    return sum + U::LEAD * some;
}
// places of all units of one head
template <class U>
__device__ __forceinline__ int head_span(const AttnArgs& a, const Segment& g) {
    if (g.n == 0) return 0;
    const int nu = U::count(a, g);
    return span_before<U>(a, g, nu, nu);
}

// A line of N places is cut into shares of q = max(ceil(N / CTAs), least); CTA c has [c q, (c + 1) q).  A least
// share, because a piece costs its prologue and a join.  On the tcgen05 line every unit has LEAD empty places in front of its tiles, so
// that a share of many short units is no longer than one of few long ones (prompts of 8001 tokens: shares of 210 tiles in 5 to 12
// units ended between 360 and 405 us).
__device__ __forceinline__ int share_tiles(int N, int ctas, int least) { return max((int)(((int64_t)N + ctas - 1) / ctas), least); }
// Least share of the few-row line.  Where there is less work than CTAs, q tiles to a share take about 0.62 q us, and the t / q pieces of a
// row whose keys are t tiles 0.85 us for every 16 in the join: the sum is least at q = sqrt(0.086 t).  t is taken as the mean over the
// segments.  One request of 100 / 300 / 600 / 1500 / 4000 keys, 8 heads of 128 channels, from CUDA graphs on three inputs in turn:
// 10.3 / 10.3 / 11.7 / 14.4 / 16.4 us; with four tiles for all 12.4 / 13.0 / 13.6 / 14.4 / 16.4, with one for all 10.3 / 10.3 / 12.3 / 14.5 / 18.6.
// (The constants are those of 128 channels; other head sizes and counts were not tuned for.)
__device__ __forceinline__ int few_min_tiles(const AttnArgs& a, int n) {
    return max((int)(sqrtf(0.086f * (float)n / ((float)(a.P + a.R) * (float)FewUnits::heads(a))) + 0.5f), 1);
}
constexpr int AT_WIDE_MIN_TILES = 4;
__device__ __forceinline__ int wide_share(const AttnArgs& a, int N, int ctas) { return share_tiles(N, ctas, AT_WIDE_MIN_TILES * (a.mask ? 2 : 1)); }
// Shares of the two lines of a step that has both (nf, nw tiles).  The tcgen05 kernel is bound by arithmetic, the few-row kernel by
// memory, and both are resident at once: the first gets as many CTAs as its part of the SMs' time, the second runs on the other
// SMs.  With 128 channels and the other kernel beside it, a place on the tcgen05 line takes an SM about 1.75 us (1.3, 2560 cycles, where it has
// the machine to itself), a few-row tile 0.6 us: three to one.  (256 requests behind 16384 keys when this was chosen: 150 us like this, 170 us with
// all SMs on one kernel after the other; 66 tcgen05 CTAs 150, 50 181, 84 157.  64 channels were not tuned for.)  How long either takes is only known that roughly, so the
// few-row shares are several rounds of the SMs left over: those that the tcgen05 kernel leaves early take from the last round.
__device__ __forceinline__ void share_lines(const AttnArgs& a, int nf, int nw, int32_t* share) {
    const int sms = a.wide_ctas;
    int wide = sms, few = min(a.few_ctas, 2 * sms);
    // With a mask a tile has two places, or three with both row tiles: 0.4 of a tile to a place.  (Small drafts behind a prefix, 0.25 / 0.4 / 0.65 / 1: 64 of 2
    // tokens behind 16000 + 1000 keys 106 / 96 / 103 / 105 us, 200 of 3 behind 2000 + 800 174 / 155 / 152 / 181, 96 of 3 behind 4000 + 500 88 / 86 / 87 / 92,
    // 32 of 3 behind 4000 + 300 47 / 50 / 50 / 50.)
    const float tiles = a.mask ? 0.4f * nw : (float)nw;
    if (nf > 0 && nw > 0) wide = max((int)(sms * (3.0f * tiles) / (3.0f * tiles + nf) + 0.5f), 1);
    const int q = wide_share(a, nw, wide);
    const int left = 2 * (sms - (nw + q - 1) / q);
    if (nw > 0 && left > 0 && left <= a.few_ctas) few = a.few_ctas / left * left;
    share[0] = share_tiles(nf, few, few_min_tiles(a, nf));
    share[1] = q;
}

// Where a cursor finds segments and their first tiles: what the plan kernel left in the workspace, or (SELF) shared memory.
template <bool SELF>
struct LineSource {
    const Segment* seg;
    const int32_t* start;
    __device__ __forceinline__ int begin(int s) const { return SELF ? start[s] : load_plan(start + s); }
    __device__ __forceinline__ Segment load(int s) const {
        if (SELF) return seg[s];
        Segment g;
        const int4* src = reinterpret_cast<const int4*>(seg + s);
        reinterpret_cast<int4*>(&g)[0] = __ldcg(src);
        reinterpret_cast<int4*>(&g)[1] = __ldcg(src + 1);
        return g;
    }
};

// A position on a line: key tile kt of unit u of head (group) h of segment s; after seek, kt < 0 where it lies in front of the unit's tiles.
template <class U, bool SELF = false>
struct Cursor {
    int s, h, u, kt, nu, nt;
    Segment g;
    // all lanes of a warp together
    __device__ void seek(const AttnArgs& a, const LineSource<SELF>& src, int S, int x) {
        const int lane = threadIdx.x & 31;
        int lo = 0, len = S;
        while (len > 1) {                // the last segment that begins at or before x, 32 candidates at a time
            const int step = (len + 31) / 32, i = lane * step;
            const uint32_t b = __ballot_sync(0xFFFFFFFFu, i < len && src.begin(lo + i) <= x);
            const int k = 31 - __clz(b);
            lo += k * step;
            len = min(step, len - k * step);
        }
        s = lo;
        g = src.load(s);
        nu = U::count(a, g);
        int y = x - g.start;
        h = y / g.tiles;
        y -= h * g.tiles;
        if (!(g.flags & SEG_OWN)) {
            nt = unit_tiles<U>(a, g, 0);
            const int span = unit_span<U>(nt, U::weight(a, g, 0));
            u = min(y / span, nu - 1);
            const int w = U::weight(a, g, u);
            kt = (y - u * span) / w - U::LEAD;               // a tile counts where its last place is
        } else if (nu <= AT_LOOP_UNITS) {
            u = 0;
            nt = unit_tiles<U>(a, g, 0);
            while (y >= unit_span<U>(nt, 1)) {
                y -= unit_span<U>(nt, 1);
                nt = unit_tiles<U>(a, g, ++u);
            }
            kt = y - U::LEAD;
        } else {
            int b = 0, e = nu;           // the last unit with at most y places before it
            while (e - b > 1) {
                const int mid = (b + e) >> 1;
                if (span_before<U>(a, g, nu, mid) <= y) b = mid; else e = mid;
            }
            u = b;
            nt = unit_tiles<U>(a, g, u);
            kt = y - span_before<U>(a, g, nu, u) - U::LEAD;
        }
    }
    // to the first tile of the next unit that has any; the caller knows that one exists
    __device__ void next_unit(const AttnArgs& a, const LineSource<SELF>& src, int line) {
        kt = 0;
        do {
            if (++u == nu) {
                u = 0;
                if (++h == U::heads(a)) {
                    h = 0;
                    do g = src.load(++s); while (g.tiles == 0 || (g.flags & SEG_WIDE) != line);
                    nu = U::count(a, g);
                }
            }
            nt = unit_tiles<U>(a, g, u);
        } while (nt == 0);
    }
};

// (last) place of the first tile of unit u of head h of a segment
template <class U>
__device__ __forceinline__ int unit_begin(const AttnArgs& a, const Segment& g, int h, int u) {
    return g.start + h * g.tiles + span_before<U>(a, g, U::count(a, g), u) + (U::LEAD + 1) * U::weight(a, g, u) - 1;
}

// unit_x0: (last) place of the unit's first tile
__device__ __forceinline__ void tell_cut(CutUnit* c, int unit_x0, int tiles, int weight, int x0, int x1, int q, int h, int u,
                                         const Segment& g) {
    c->begin = unit_x0;
    c->weight = weight;
    c->share = q;
    c->h = h;
    c->u = u;
    c->t0 = g.t0;
    c->n = g.n;
    c->tiles = unit_x0 + (tiles - 1) * weight >= x1 && unit_x0 >= x0 && !(g.flags & SEG_TWO) ? tiles : 0;
}

// ------------------------------------------------------------------------------------------------ the plan
// Inclusive sum over the block of one pair of values per thread; s_warp: [2][32] in shared memory.  Returns the block's totals in `total`.
__device__ __forceinline__ void block_scan2(int (&v)[2], int (&total)[2], int (*s_warp)[32], int warps) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xFFFFFFFFu, v[j], o);
            if (lane >= o) v[j] += up;
        }
        if (lane == 31) s_warp[j][warp] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int x = lane < warps ? s_warp[j][lane] : 0;
        int inc = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xFFFFFFFFu, inc, o);
            if (lane >= o) inc += up;
        }
        total[j] = __shfl_sync(0xFFFFFFFFu, inc, 31);
        v[j] += __shfl_sync(0xFFFFFFFFu, inc - x, warp);
    }
    __syncthreads();
}

// Rows without any key (fewer own keys than new tokens, and no prefix) are in no unit, or in one that has other rows: 0, -inf.
// One warp, for tokens [t0, t0 + n).
__device__ __forceinline__ void clear_rows(const AttnArgs& a, int t0, int n) {
    const int lane = threadIdx.x & 31;
    for (int t = t0; t < t0 + n; ++t) {
        for (int c = lane; c < a.Hq * a.head_dim / 8; c += 32) *reinterpret_cast<uint4*>(a.o + (int64_t)t * a.ldo + c * 8) = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse)
            for (int c = lane; c < a.Hq; c += 32) a.lse[(int64_t)t * a.Hq + c] = -INFINITY;
    }
}

// One CTA of up to 1024 threads, a thread per segment; lengths are read once, groups are searched in shared memory.
constexpr int AT_PLAN_GROUPS = 512;    // groups of a step that fit there; more are looked up in global memory

__global__ void __launch_bounds__(1024) attn_plan_kernel(const AttnArgs a) {
    __shared__ int s_warp[2][32];
    __shared__ int s_off[AT_PLAN_GROUPS + 1], s_len[AT_PLAN_GROUPS], s_mixed[AT_PLAN_GROUPS];
    grid_launch_dependents();
    grid_dependency_wait();
    const int tid = threadIdx.x, threads = blockDim.x, S = a.P + a.R;
    const bool in_smem = a.P <= AT_PLAN_GROUPS;
    auto off = [&](int g) { return in_smem ? s_off[g] : attn_group(a, g); };
    auto len = [&](int g) { return in_smem ? s_len[g] : attn_keys(a.prefix_len[g], a.pcols, a.page_shift); };
    // the last group that begins at or before request r, if the request is in it and its prefix is not empty
    auto group_of = [&](int r) -> int {
        if (a.P == 0) return -1;
        int lo = 0, hi = a.P;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (off(mid) <= r) lo = mid; else hi = mid;
        }
        return off(lo) <= r && r < off(lo + 1) && len(lo) > 0 ? lo : -1;
    };
    if (a.P > 0) {
        if (in_smem) {
            for (int g = tid; g <= a.P; g += threads) {
                s_off[g] = attn_group(a, g);
                if (g < a.P) {
                    s_len[g] = attn_keys(a.prefix_len[g], a.pcols, a.page_shift);
                    s_mixed[g] = 0;
                }
            }
            __syncthreads();
            // groups that have requests with few rows need a prefix segment (with more groups than fit here all have one)
            for (int s = tid; s < S; s += threads) {
                const int r = s - a.P;
                if (r < 0) continue;
                const int rows = (attn_row(a, r + 1) - attn_row(a, r)) * a.G;
                if (rows > 0 && (rows < AT_MERGE_ROWS || rows < a.wide_min_rows)) {
                    const int g = group_of(r);
                    if (g >= 0) s_mixed[g] = 1;
                }
            }
            __syncthreads();
        }
    }
    auto mixed = [&](int g) { return in_smem ? s_mixed[g] != 0 : true; };
    int carry[2] = {0, 0};
    bool two = false, empty = false, longer = false, falls = false;
    for (int s0 = 0; s0 < S; s0 += threads) {
        const int s = s0 + tid;
        int own[2] = {0, 0}, inc[2], total[2];
        Segment g;
        if (s < S) {
            g.plen = 0;
            g.flags = s >= a.P && !a.mask ? SEG_OWN : 0;
            if (s < a.P) {
                const int r0 = off(s), r1 = max(off(s + 1), r0);
                falls |= off(s + 1) < r0;
                g.klen = len(s);
                g.t0 = attn_row(a, r0);
                g.n = g.klen > 0 && mixed(s) ? max(attn_row(a, r1) - g.t0, 0) : 0;
                g.group = s;
                g.flags = SEG_TWO;
            } else {
                const int r = s - a.P;
                g.t0 = attn_row(a, r);
                g.n = attn_row(a, r + 1) - g.t0;
                falls |= g.n < 0;
                g.n = max(g.n, 0);
                g.klen = attn_keys(a.kv_len[r], a.cols, a.page_shift);
                g.group = group_of(r);
                if (g.group >= 0) {
                    if (mixed(g.group)) g.flags |= SEG_TWO;
                    else g.plen = len(g.group);
                }
                two |= g.n > 0 && (g.flags & SEG_TWO);
                empty |= g.group < 0 && seg_blind(a, g) > 0;
                if (a.P > 0 && g.n <= 32)          // the tokens' requests; of longer ones and behind the last token further down
                    for (int t = g.t0; t < g.t0 + g.n; ++t) a.plan.tok_req[t] = g.flags & SEG_TWO ? r : -1;
                longer |= a.P > 0 && g.n > 32;
            }
            if (g.n * a.G >= a.wide_min_rows) {
                g.flags |= SEG_WIDE;
                g.tiles = head_span<WideUnits>(a, g);
                own[1] = g.tiles * WideUnits::heads(a);
            } else {
                g.tiles = head_span<FewUnits>(a, g);
                own[0] = g.tiles * FewUnits::heads(a);
            }
        }
        inc[0] = own[0];
        inc[1] = own[1];
        block_scan2(inc, total, s_warp, threads / 32);
        if (s < S) {
            const int few = carry[0] + inc[0] - own[0], wide = carry[1] + inc[1] - own[1];
            a.plan.few_start[s] = few;
            a.plan.wide_start[s] = wide;
            g.start = g.flags & SEG_WIDE ? wide : few;
            a.plan.seg[s] = g;
        }
        carry[0] += total[0];
        carry[1] += total[1];
    }
    two = __syncthreads_or(two);
    empty = __syncthreads_or(empty || longer || falls);
    // Offsets that fall: requests or groups may hold the same rows, and all their tiles together pass what the host has counted.
    if (empty && __syncthreads_or(falls)) {
        two = empty = false;
        carry[0] = carry[1] = 0;
    }
    if (tid == 0) {
        a.plan.share[2] = two;
        a.plan.few_start[S] = carry[0];
        a.plan.wide_start[S] = carry[1];
        share_lines(a, carry[0], carry[1], a.plan.share);
    }
    if (two)
        for (int t = attn_row(a, a.R) + tid; t < a.T; t += threads) a.plan.tok_req[t] = -1;
    if (empty) {
        for (int r = tid >> 5; r < a.R; r += threads / 32) {
            const Segment& g = a.plan.seg[a.P + r];
            if (g.group < 0) clear_rows(a, g.t0, seg_blind(a, g));
            if (two && g.n > 32)
                for (int t = g.t0 + (tid & 31); t < g.t0 + g.n; t += 32) a.plan.tok_req[t] = g.flags & SEG_TWO ? r : -1;
        }
    }
}

// ------------------------------------------------------------------------------------------------ pieces
struct PieceList {           // pieces of one row from one unit
    int count;               // 0: none; 1: the whole unit
    int first, rest, stride; // rows of the partial results: `first` for piece 0, rest + i * stride for the others
};
// A unit of `tiles` tiles of `weight` places from `begin` on, cut into shares of q (each of which has a tile at least); `base`: row of the line's slots; stride: rows between two
// slots of a CTA; row: row in a slot; whole: row of the dense results
__device__ __forceinline__ PieceList list_pieces(int begin, int tiles, int weight, int q, int base, int stride, int row, int whole) {
    PieceList p;
    const int c0 = begin / q, c1 = (begin + (tiles - 1) * weight) / q;
    p.count = c1 - c0 + 1;
    p.stride = 2 * stride;
    p.rest = base + c0 * 2 * stride + row;
    p.first = p.count == 1 ? whole : p.rest + (begin > c0 * q ? stride : 0);
    return p;
}

// (m, l) of a piece as the join reads it.  NaN scores leave the maximum alone (a maximum drops NaN), but not the sum.  Such a piece says
// m = +inf: the join then weighs it with NaN and all others with 0, where a maximum of -inf, or far below the others', would drop it.
__device__ __forceinline__ float2 piece_ml(float m, float l) { return make_float2(l != l ? INFINITY : m, l); }

// --------------------------------------------------------------------------------------------- few rows
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool valid, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0), "l"(policy) : "memory");
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

constexpr int FEW_SELF = 256;          // requests whose line every CTA lays out for itself

template <int D, int HW, bool SELF>
struct FewCfg {
    static constexpr int KV_BYTES = 16 * D * 2;                  // one warp's 16 keys (or values) of a tile
    static constexpr int SLOT_BYTES = 2 * KV_BYTES;
    static constexpr int STAGES = D == 128 ? 3 : 6;
    static constexpr int RING = 4 * STAGES * SLOT_BYTES;         // every warp has its own ring
    static constexpr int JOIN_FLOATS = 16 * D + 32;              // one warp's O, m and l
    static constexpr int JOIN = HW < 4 ? 2 * JOIN_FLOATS * 4 : 0;
    static constexpr int PLAN = SELF ? FEW_SELF * (int)sizeof(Segment) + FEW_SELF * 4 : 0;
    static constexpr int SMEM = RING + JOIN + PLAN;
};

// One CTA: four warps, each with its own ring of cp.async slots and its own (m, l, O), so that no barrier runs inside the
// key loop.  With four heads to a unit a warp has a head and no barrier runs at all; the four heads of a token lie side by side
// in the cache, so the CTA still reads whole 1 KB rows.  Where the number of heads is not a multiple of four, two or four warps
// take different keys of a head and are joined through shared memory at the end of a unit.  (All warps on one head
// whatever the head count: 129 us for 256 requests of ~512 keys, 80 like this; the join took three barriers a unit.)
// HBM bounds it: 7 requests of 29572 keys 70 us, 6.05 TB/s.
// It needs nothing of the tcgen05 kernel that may be launched in front of it, so it begins (`early`) on every SM that has no
// tcgen05 CTA or whose CTA has ended.  Its last CTA alone waits for that kernel before it ends: whatever comes behind waits for both,
// and no SM is held by CTAs that have nothing left to do (32 requests behind 4096 keys: 43 -> 38 us).
// Without prefixes and prompts, up to FEW_SELF requests, with a multiple of four key/value heads, every CTA lays out the line for itself in
// shared memory (SELF) and no plan kernel runs: the launch and its two trips through L2 would be a third of the smallest calls.  (With other
// head counts the warps' join buffers would come on top: 124 KB for one head of 128 channels, one CTA to an SM instead of two.)
// The loads run on over the ends of units.  A page number is fetched one tile ahead of the loads that need it.
// TREE: new tokens are seen by the bits of a mask, looked up only for the tiles that hold some.
template <int D, int HW, bool SELF, bool TREE>
__global__ void __launch_bounds__(AT_FEW_THREADS, 2) attn_few_kernel(const AttnArgs a, bool early) {
    using C = FewCfg<D, HW, SELF>;
    constexpr int NJ = D / 8;          // 8-channel column blocks of O
    constexpr int KS = D / 16;         // k steps of Q K^T
    constexpr int CHUNKS = D / 8;      // 16-byte chunks of a key
    constexpr int KEYS = 64 / HW;      // keys of a tile
    extern __shared__ __align__(128) uint8_t at_smem[];
    grid_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (!early) grid_dependency_wait();
    const int S = a.P + a.R;
    LineSource<SELF> src = {a.plan.seg, a.plan.few_start};
    int N, q;
    if (SELF) {
        __shared__ int s_warp[2][32];
        Segment* seg = reinterpret_cast<Segment*>(at_smem + C::RING + C::JOIN);
        int* start = reinterpret_cast<int*>(seg + FEW_SELF);
        int carry = 0;
        bool empty = false, falls = false;
        for (int s0 = 0; s0 < S; s0 += AT_FEW_THREADS) {
            const int s = s0 + threadIdx.x;
            int inc[2] = {0, 0}, total[2], own = 0;
            if (s < S) {
                Segment g;
                g.plen = 0;
                g.flags = TREE ? 0 : SEG_OWN;
                g.group = -1;
                g.t0 = attn_row(a, s);
                g.n = attn_row(a, s + 1) - g.t0;
                falls |= g.n < 0;
                g.n = max(g.n, 0);
                g.klen = attn_keys(a.kv_len[s], a.cols, a.page_shift);
                g.tiles = head_span<FewUnits>(a, g);
                own = g.tiles * FewUnits::heads(a);
                inc[0] = own;
                seg[s] = g;
                empty |= seg_blind(a, g) > 0;
            }
            block_scan2(inc, total, s_warp, AT_FEW_THREADS / 32);
            if (s < S) start[s] = seg[s].start = carry + inc[0] - own;
            carry += total[0];
        }
        empty = __syncthreads_or(empty || falls);
        N = carry;
        if (empty && __syncthreads_or(falls)) {    // as in the plan kernel
            empty = false;
            N = 0;
        }
        q = share_tiles(N, a.few_ctas, few_min_tiles(a, N));
        src.seg = seg;
        src.start = start;
        if (empty)
            for (int r = blockIdx.x * 4 + warp; r < S; r += gridDim.x * 4)
                clear_rows(a, seg[r].t0, seg_blind(a, seg[r]));
    } else {
        N = load_plan(a.plan.few_start + S);
        q = load_plan(a.plan.share);
    }
    const int x0 = (int)min((int64_t)q * blockIdx.x, (int64_t)N), x1 = (int)min((int64_t)x0 + q, (int64_t)N);
    if (x0 >= x1) {
        if (threadIdx.x == 0) a.plan.cut[0][blockIdx.x].tiles = 0;
        if (early && blockIdx.x == gridDim.x - 1) grid_dependency_wait();
        return;
    }

    const uint32_t ring = smem_u32(at_smem) + warp * C::STAGES * C::SLOT_BYTES;
    float* join = reinterpret_cast<float*>(at_smem + C::RING);

    Cursor<FewUnits, SELF> cur, ld;
    cur.seek(a, src, S, x0);
    ld = cur;
    const int page_mask = (1 << a.page_shift) - 1;
    const int hw = warp % HW;          // head of the warp inside the unit
    const int kw = warp / HW * 16;     // first key of the warp inside a tile
    // page that holds the warp's 16 keys of the loader's tile (a page has at least 16 tokens)
    auto page_of = [&]() -> int {
        const int key = ld.kt * KEYS + kw;
        if (key >= ld.g.klen) return -1;
        const int p = seg_pages(a, ld.s)[key >> a.page_shift];     // klen is within the list's columns
        return (p >= 0 && p < a.n_pages) ? p : -1;
    };
    int xl = x0;                       // loader's position
    int page = page_of();
    const uint64_t policy = l2_policy_evict_first();   // read once: must not push code, plan and partial results out of L2
    auto load = [&](int slot) {
        if (xl < x1) {
            const int key = ld.kt * KEYS + kw;
            const int64_t base = (int64_t)max(page, 0) * a.page_stride + (int64_t)(key & page_mask) * a.token_stride +
                                 (int64_t)(ld.h * HW + hw) * a.head_stride;
            const uint32_t dst = ring + slot * C::SLOT_BYTES;
            const int nvalid = page >= 0 ? ld.g.klen - key : 0;   // keys past the end (and absent pages) read as zero
#pragma unroll
            for (int i = 0; i < 16 * CHUNKS / 32; ++i) {
                const int r = (i * 32 + lane) / CHUNKS, c = (i * 32 + lane) % CHUNKS;
                const int64_t off = r < nvalid ? base + (int64_t)r * a.token_stride + c * 8 : 0;
                const uint32_t d = dst + r * (D * 2) + ((c ^ (r & 7)) * 16);
                cp_async_16(d, a.k + off, r < nvalid, policy);
                cp_async_16(d + C::KV_BYTES, a.v + off, r < nvalid, policy);
            }
            if (++xl < x1) {
                if (++ld.kt == ld.nt) ld.next_unit(a, src, 0);
                page = page_of();
            }
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < C::STAGES - 1; ++i) load(i);

    const int r0 = lane >> 2, cq = lane & 3;       // the thread's rows r0, r0 + 8 and column pair of an MMA fragment
    int slot = 0, fill = C::STAGES - 1;
    int x = x0;
    while (x < x1) {
        // ---- a unit (or the share's part of it)
        const int row0 = cur.u * AT_FEW_ROWS;
        const int nrows = min(AT_FEW_ROWS, cur.g.n * a.G - row0);
        const int head = cur.h * HW + hw;
        uint32_t qf[KS][4];
        int sees[2];
        const uint32_t* mask[2];
        const int ctx = TREE && cur.s >= a.P ? cur.g.klen - cur.g.n : 0x7FFFFFFF;      // first new token among the keys
#pragma unroll
        for (int hlf = 0; hlf < 2; ++hlf) {
            const int r = r0 + hlf * 8;
            const int tok = (row0 + r) / a.G, hd = (row0 + r) % a.G;
            const bool ok = r < nrows;
            sees[hlf] = ok ? seg_sees(cur.g, tok) : 0;
            if (TREE) mask[hlf] = a.mask + (ok ? (int64_t)(cur.g.t0 + tok) * a.ld_mask : 0);
            const uint16_t* qp = a.q + (ok ? (int64_t)(cur.g.t0 + tok) * a.ldq + (int64_t)(head * a.G + hd) * D : 0) + cq * 2;
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
        const int unit_x0 = x - cur.kt, unit_x1 = unit_x0 + cur.nt;
        const int xe = min(unit_x1, x1);
        for (; x < xe; ++x, ++cur.kt) {
            load(fill);
            if (++fill == C::STAGES) fill = 0;
            cp_async_wait<C::STAGES - 1>();
            __syncwarp();
            const uint32_t kb = ring + slot * C::SLOT_BYTES, vb = kb + C::KV_BYTES;
            const int key0 = cur.kt * KEYS + kw;
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
                const bool masked = TREE && key0 + 16 > ctx;
                uint32_t bits[2];
                if (!masked) {
#pragma unroll
                    for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + n8 * 8 + cq * 2 + (e & 1);
                            sc[n8][e] = key < sees[e >> 1] ? sc[n8][e] * a.scale_log2 : -INFINITY;
                            mx[e >> 1] = fmaxf(mx[e >> 1], sc[n8][e]);
                        }
                } else {
#pragma unroll
                    for (int hlf = 0; hlf < 2; ++hlf) bits[hlf] = tree_sees(a, mask[hlf], key0, ctx, sees[hlf]);      // sees: all keys, or none
#pragma unroll
                    for (int n8 = 0; n8 < 2; ++n8)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            sc[n8][e] = bits[e >> 1] >> (n8 * 8 + cq * 2 + (e & 1)) & 1u ? sc[n8][e] * a.scale_log2 : -INFINITY;
                            mx[e >> 1] = fmaxf(mx[e >> 1], sc[n8][e]);
                        }
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
                if (masked) {
                    // An Inf or a NaN among the values of a token would reach the rows that do not see it, through a weight of 0.  It is added
                    // here to the rows that do (any positive weight gives the same), behind the correction of O, and is 0 in the product.
                    bool odd = false;
#pragma unroll 1
                    for (int i = lane; i < 16 * CHUNKS; i += 32) odd |= has_odd(*reinterpret_cast<const uint4*>(at_smem + (vb - smem_u32(at_smem)) + i * 16));
                    if (__any_sync(0xFFFFFFFFu, odd)) {
                        uint8_t* v = at_smem + (vb - smem_u32(at_smem));
#pragma unroll 1
                        for (int k = 0; k < 16; ++k)
#pragma unroll
                            for (int j = 0; j < NJ; ++j) {
                                const uint32_t x = *reinterpret_cast<const uint32_t*>(v + k * (D * 2) + ((j ^ (k & 7)) * 16) + cq * 4);
                                const uint32_t y = x & ~drop_odd(x);       // the odd ones alone, others 0
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t z = e & 1 ? y & 0xFFFF0000u : y << 16;
                                    if ((z & 0x7F800000u) == 0x7F800000u && (bits[e >> 1] >> k & 1u)) o[j][e] += __uint_as_float(z);
                                }
                            }
                        __syncwarp();
#pragma unroll 1
                        for (int i = lane; i < 16 * CHUNKS; i += 32) {
                            uint4* x = reinterpret_cast<uint4*>(v + i * 16);
                            *x = drop_odd(*x);
                        }
                        __syncwarp();
                    }
                }
                // Weights in bf16 for P V: the tensor cores take both operands in one type, and V is bf16.  Each is off by at most 2^-8 of itself, either
                // way, as the output is from its own rounding (error of the outputs 0.0023 of their size, 0.0017 with weights in fp32); l sums them unrounded.
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
#pragma unroll
        for (int hlf = 0; hlf < 2; ++hlf) {
            l[hlf] += __shfl_xor_sync(0xFFFFFFFFu, l[hlf], 1);
            l[hlf] += __shfl_xor_sync(0xFFFFFFFFu, l[hlf], 2);
        }
        // ---- join the warps of a head: 2, 3 -> 0, 1, then (one head) 1 -> 0
#pragma unroll
        for (int step = 2; step >= HW; step >>= 1) {
            if (warp >= step && warp < 2 * step) {
                float* buf = join + (warp - step) * C::JOIN_FLOATS;
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
                const float* buf = join + warp * C::JOIN_FLOATS;
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
        if (warp < HW) {
            const bool split = unit_x0 < x0 || unit_x1 > x1;
            const bool two = cur.g.flags & SEG_TWO;
#pragma unroll
            for (int hlf = 0; hlf < 2; ++hlf) {
                const int r = r0 + hlf * 8;
                if (r >= nrows) continue;
                const int64_t token = cur.g.t0 + (row0 + r) / a.G;
                const int hq = head * a.G + (row0 + r) % a.G;
                const int64_t row = token * a.Hq + hq;
                if (!split && !two) {
                    const float inv = l[hlf] > 0.0f || l[hlf] != l[hlf] ? 1.0f / l[hlf] : 0.0f;
                    uint16_t* op = a.o + token * a.ldo + (int64_t)hq * D + cq * 2;
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        *reinterpret_cast<uint32_t*>(op + j * 8) = bf162_bits(__floats2bfloat162_rn(o[j][2 * hlf] * inv, o[j][2 * hlf + 1] * inv));
                    if (a.lse && cq == 0) a.lse[row] = l[hlf] == 0.0f ? -INFINITY : (m[hlf] + log2f(l[hlf])) * 0.69314718055994531f;
                } else {
                    const int at = split ? ((blockIdx.x * 2 + (unit_x0 > x0 ? 1 : 0)) * HW + hw) * AT_FEW_ROWS + r
                                         : dense_row(a, cur.s >= a.P, (int)row);
                    float* part = a.part + (int64_t)at * D + cq * 2;
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        *reinterpret_cast<float2*>(part + j * 8) = make_float2(o[j][2 * hlf], o[j][2 * hlf + 1]);
                    if (cq == 0) a.ml[at] = piece_ml(m[hlf], l[hlf]);
                }
            }
        }
        if (x < x1) cur.next_unit(a, src, 0);
        else if (threadIdx.x == 0) tell_cut(a.plan.cut[0] + blockIdx.x, unit_x0, unit_x1 - unit_x0, 1, x0, x1, q, cur.h, cur.u, cur.g);
    }
    cp_async_wait<0>();
    if (early && blockIdx.x == gridDim.x - 1) grid_dependency_wait();
}

// ------------------------------------------------------------------------------------------------- join
// Joins the pieces of rows whose keys were not all in one unit of one share, in the order of the lines (so the result does not depend on
// which CTA was first), one warp to a row.  Two kinds of blocks, because the rows to be joined are not known on the host and looking at
// every row costs more than the joining (262 us for 8001 tokens of prompts against 1 ms of attention, when it was done that way):
//   units that the end of a share cuts, as the attention kernels told them: blocks for every share of either line;
//   rows with two sources (prefix and own keys): blocks over the tokens, only launched where there are prefixes.
// The code is kept short and mostly rolled: behind a kernel that has streamed hundreds of MB through L2 it comes from HBM line by
// line, and a version with four rows to a warp and pieces shared out over warps, though it had more loads under way, took longer.
constexpr int AT_JOIN_THREADS = 256;
constexpr int AT_JOIN_WARPS = AT_JOIN_THREADS / 32;

// FLIGHT: pieces under way at a time.  16 (two blocks to an SM) where the step has few rows, whose keys are in many pieces each; 8
// (three blocks) where there are many rows (7 requests of 29572 keys: 82.9 us with 16, 86.7 with 8; prompts of 8001 tokens 454 and 443).
template <int D, int FLIGHT>
__device__ __forceinline__ void join_row(const AttnArgs& a, const PieceList (&p)[2], int token, int hq) {
    constexpr int V = D / 32;          // channels per lane
    const int lane = threadIdx.x & 31;
    const float* part = a.part + lane * V;
    float m = -INFINITY, l = 0.0f, o[V];
#pragma unroll
    for (int y = 0; y < V; ++y) o[y] = 0.0f;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const int n = which ? p[1].count : p[0].count, first = which ? p[1].first : p[0].first;
        const int rest = which ? p[1].rest : p[0].rest, stride = which ? p[1].stride : p[0].stride;
#pragma unroll 1
        for (int i = 0; i < n; i += FLIGHT) {
            float2 ml[FLIGHT];
            float v[FLIGHT][V];
#pragma unroll
            for (int j = 0; j < FLIGHT; ++j) {
                ml[j] = make_float2(-INFINITY, 0.0f);
                if (i + j < n) {
                    const int at = i + j ? rest + (i + j) * stride : first;
                    ml[j] = a.ml[at];
                    const float* src = part + (int64_t)at * D;
                    if (V == 4) {
                        const float4 q = *reinterpret_cast<const float4*>(src);
                        v[j][0] = q.x; v[j][1] = q.y; v[j][V - 2] = q.z; v[j][V - 1] = q.w;
                    } else {
                        const float2 q = *reinterpret_cast<const float2*>(src);
                        v[j][0] = q.x; v[j][1] = q.y;
                    }
                }
            }
            float mn = m;
#pragma unroll
            for (int j = 0; j < FLIGHT; ++j) mn = fmaxf(mn, ml[j].x);
            if (mn == -INFINITY) continue;
            const float f = exp2_approx(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int y = 0; y < V; ++y) o[y] *= f;
#pragma unroll
            for (int j = 0; j < FLIGHT; ++j) {
                const float w = exp2_approx(ml[j].x - mn);
                if (w != 0.0f) {           // a piece without weight may hold anything
                    l = fmaf(ml[j].y, w, l);
#pragma unroll
                    for (int y = 0; y < V; ++y) o[y] = fmaf(v[j][y], w, o[y]);
                }
            }
        }
    }
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    uint16_t* op = a.o + (int64_t)token * a.ldo + (int64_t)hq * D + lane * V;
    if (V == 4)
        *reinterpret_cast<uint2*>(op) = make_uint2(bf162_bits(__floats2bfloat162_rn(o[0] * inv, o[1] * inv)),
                                                   bf162_bits(__floats2bfloat162_rn(o[V - 2] * inv, o[V - 1] * inv)));
    else
        *reinterpret_cast<uint32_t*>(op) = bf162_bits(__floats2bfloat162_rn(o[0] * inv, o[1] * inv));
    if (a.lse && lane == 0) a.lse[(int64_t)token * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// Blocks in this order: those with the longest chains come first, the many that mostly find nothing to do last.
struct JoinGrid {
    int row_blocks;          // over the tokens' rows
    int wide_blocks;         // over the parts, 1 << wide_split of them, of the 256 rows of a cut wide unit: a block for every part that there can be, or
                             // (WALK) fewer, that share out the parts that there are
    int wide_split;
    int few_split;           // few_ctas << few_split blocks: a part of the rows of a cut few-row unit each
};

constexpr int64_t AT_JOIN_FEW_ROWS = 4096;     // between 224 and 256032 rows of the two steps above
template <int D, int FLIGHT, bool WALK>
__global__ void __launch_bounds__(AT_JOIN_THREADS, FLIGHT > 8 ? 2 : 3) attn_join_kernel(const AttnArgs a, const JoinGrid grid) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int warp = threadIdx.x >> 5;
    int b = blockIdx.x;
    PieceList p[2];
    p[0].count = p[0].first = p[0].rest = p[0].stride = 0;
    if (b >= grid.row_blocks) {
        b -= grid.row_blocks;
        const bool wide = b < grid.wide_blocks;
        if (!wide) b -= grid.wide_blocks;
        const int split = wide ? grid.wide_split : grid.few_split;
        const int slot_rows = wide ? 2 * AT_WIDE_TILE : a.few_hw * AT_FEW_ROWS, rows = slot_rows >> split;
#pragma unroll 1
        for (int part = b;; part += grid.wide_blocks) {
            int c = part >> split;               // CTA that told the unit
            if (WALK && wide) {                  // the (part >> split)-th of those that told one
                constexpr int WORDS = (AT_WIDE_CTAS + 31) / 32;
                int tiles[WORDS], n = c;
                c = -1;
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    const int at = i * 32 + (threadIdx.x & 31);
                    tiles[i] = at < a.wide_ctas ? a.plan.cut[1][at].tiles : 0;
                }
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    uint32_t told = __ballot_sync(0xFFFFFFFFu, tiles[i] != 0);
                    const int k = __popc(told);
                    if (c < 0 && n < k) {
                        for (; n > 0; --n) told &= told - 1;
                        c = i * 32 + __ffs((int)told) - 1;
                    }
                    n -= k;
                }
                if (c < 0) return;
            }
            const CutUnit cut = a.plan.cut[wide][c];
            if (cut.tiles == 0) return;
            const int row0 = (part & ((1 << split) - 1)) * rows;
            const PieceList list = list_pieces(cut.begin, cut.tiles, cut.weight, cut.share, wide ? AT_FEW_SLOTS : 0, slot_rows, 0, 0);      // two pieces at least
#pragma unroll 1
            for (int i = warp; i < rows; i += AT_JOIN_WARPS) {
                const int row = row0 + i, r = wide ? row % AT_WIDE_TILE : cut.u * AT_FEW_ROWS + row % AT_FEW_ROWS;
                const int tok = r / a.G + (wide ? (cut.u * 2 + row / AT_WIDE_TILE) * a.tpt : 0);
                if ((wide && r >= a.tpt * a.G) || tok >= cut.n) continue;
                p[1] = list;
                p[1].first += row;
                p[1].rest += row;
                join_row<D, FLIGHT>(a, p, cut.t0 + tok, (wide ? cut.h : cut.h * a.few_hw + row / AT_FEW_ROWS) * a.G + r % a.G);
            }
            if (!WALK || !wide) return;
        }
    }
    // rows that have a prefix and own keys
    const int two = a.plan.share[2], nf = a.plan.share[0], nw = a.plan.share[1], rows = a.T * a.Hq;
    if (two == 0) return;
#pragma unroll 1
    for (int i = b * AT_JOIN_WARPS + warp; i < rows; i += grid.row_blocks * AT_JOIN_WARPS) {
        const int t = i / a.Hq, hq = i - t * a.Hq, h = hq / a.G, g = hq - h * a.G;
        const int r = a.plan.tok_req[t];
        if ((unsigned)r >= (unsigned)a.R) continue;
        // a token that no request covers holds what the workspace held before: it counts only inside its request
        const Segment own = a.plan.seg[a.P + r];
        if (t < own.t0 || t >= own.t0 + own.n || !(own.flags & SEG_TWO)) continue;
        // even lanes work out the pieces of the prefix, odd lanes those of the own keys
        const int which = threadIdx.x & 1;
        const Segment sg = which ? own : a.plan.seg[own.group];
        const int tok = t - sg.t0, fr = tok * a.G + g;
        PieceList x;
        x.count = x.first = x.rest = x.stride = 0;
        if (tok >= 0 && tok < sg.n) {
            const bool w = sg.flags & SEG_WIDE;
            const int tpt = a.tpt, u = w ? tok / (2 * tpt) : fr / AT_FEW_ROWS, in = tok - u * 2 * tpt, hs = a.few_hw == 4 ? 2 : a.few_hw == 2 ? 1 : 0;
            const int row = w ? (in >= tpt ? AT_WIDE_TILE + (in - tpt) * a.G : in * a.G) + g : (h & (a.few_hw - 1)) * AT_FEW_ROWS + fr % AT_FEW_ROWS;
            const int nt = w ? unit_tiles<WideUnits>(a, sg, u) : unit_tiles<FewUnits>(a, sg, u);
            const int begin = w ? unit_begin<WideUnits>(a, sg, h, u) : unit_begin<FewUnits>(a, sg, h >> hs, u);
            if (nt) x = list_pieces(begin, nt, w ? WideUnits::weight(a, sg, u) : 1, w ? nw : nf, w ? AT_FEW_SLOTS : 0, w ? 2 * AT_WIDE_TILE : a.few_hw * AT_FEW_ROWS, row, dense_row(a, which, i));
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            p[k].count = __shfl_sync(0xFFFFFFFFu, x.count, k);
            p[k].first = __shfl_sync(0xFFFFFFFFu, x.first, k);
            p[k].rest = __shfl_sync(0xFFFFFFFFu, x.rest, k);
            p[k].stride = __shfl_sync(0xFFFFFFFFu, x.stride, k);
        }
        join_row<D, FLIGHT>(a, p, t, hq);
    }
}

}  // namespace osc
