// Kernels around a paged key/value cache, between the QKV projection and the attention:
//   kv_slots_kernel     pages for the new tokens of every request, slots and positions of the tokens
//   qk_norm_rope_kernel RMSNorm of the query and key heads, rotation by position, keys and values into the cache
#include <algorithm>

#include "common.cuh"

namespace osc {

// ---------------------------------------------------------------------------------------------- kv_slots
// Request r holds `cached` tokens and gets `fresh` new ones.  With have = ceil(cached / p) and
// want = ceil((cached + fresh) / p) pages, it takes want - have pages from the free list, in request order:
//   first_r      = sum over r' < r of (want - have)
//   table[r][have + j] = free[first_r + j]
//   row_off      = exclusive sum of fresh
//   token i of r : at = cached + i, slot = table[r][at / p] * p + at % p, position = base + at
// Both sums run over the requests only, so every CTA does them for itself (32-bit halves of one 64-bit value that stop at
// 2^31 - 1, shuffle scans) instead of a second launch; tokens and pages are then shared out over the grid, each finding its
// request by binary search in shared memory.  A page that this call hands out is read from the free list, not
// from the table, so nothing written by another CTA is read.  What bounds it is latency: lengths -> scan ->
// search -> page -> store, one after the other.

struct KvSlotsArgs {
    const int32_t* cached;
    const int32_t* fresh;
    const int32_t* base;    // may be null: 0
    const int32_t* free_pages;
    int32_t* table;
    int64_t ld_table;
    int32_t* row_off;
    int32_t* kv_len;
    int32_t* slots;
    int32_t* positions;
    int32_t* taken;
    int R, page, n_free, cols, T;
};

// largest i in [0, n) with start[i] <= x (start ascending, start[0] <= x)
__device__ __forceinline__ int search_last(const int* start, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// ceil(n / page) for 0 <= n < 2^31: the sum passes 31 bits, but not 32
__device__ __forceinline__ int pages_of(int n, int page) { return (int)(((unsigned)n + (unsigned)page - 1u) / (unsigned)page); }

// Tokens in the low half, pages in the high half.  Lengths are the caller's: a half that has reached 2^31 - 1 stays there (none of the
// first T tokens, and no page of the list, lies behind it).  Grouping does not matter to a sum that stops, so it can be scanned.
__device__ __forceinline__ unsigned long long add_counts(unsigned long long a, unsigned long long b) {
    const unsigned lo = min((unsigned)a + (unsigned)b, 0x7FFFFFFFu), hi = min((unsigned)(a >> 32) + (unsigned)(b >> 32), 0x7FFFFFFFu);
    return (unsigned long long)lo | (unsigned long long)hi << 32;
}

// KS_THREADS: 256, or 1024 for more requests than that, so that nearly every step is one chunk of requests
template <int KS_THREADS>
__global__ void __launch_bounds__(KS_THREADS) kv_slots_kernel(const KvSlotsArgs a) {
    __shared__ int s_row[KS_THREADS + 1], s_first[KS_THREADS + 1], s_cached[KS_THREADS], s_base[KS_THREADS];
    __shared__ unsigned long long s_warp[KS_THREADS / 32];
    grid_launch_dependents();
    grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned long long carry = 0;   // tokens in the low half, pages in the high half, of the requests before the chunk
    for (int r0 = 0; r0 < a.R; r0 += KS_THREADS) {
        const int nr = min(KS_THREADS, a.R - r0);
        int cached = 0, fresh = 0, need = 0;
        if (tid < nr) {
            cached = max(a.cached[r0 + tid], 0);
            fresh = max(a.fresh[r0 + tid], 0);
            need = (int)(((long long)cached + fresh + a.page - 1) / a.page - ((long long)cached + a.page - 1) / a.page);
            s_cached[tid] = cached;
            s_base[tid] = a.base ? a.base[r0 + tid] : 0;
        }
        unsigned long long inc = (unsigned long long)(unsigned)fresh | (unsigned long long)(unsigned)need << 32;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xFFFFFFFFu, inc, o);
            if (lane >= o) inc = add_counts(inc, up);
        }
        if (lane == 31) s_warp[warp] = inc;
        unsigned long long exc = __shfl_up_sync(0xFFFFFFFFu, inc, 1);
        __syncthreads();
        unsigned long long before = carry, total = carry;
#pragma unroll 1
        for (int w = 0; w < KS_THREADS / 32; ++w) {
            if (w < warp) before = add_counts(before, s_warp[w]);
            total = add_counts(total, s_warp[w]);
        }
        exc = lane ? add_counts(before, exc) : before;
        s_row[tid] = (int)(unsigned)exc;
        s_first[tid] = (int)(exc >> 32);
        if (tid == 0) {
            s_row[KS_THREADS] = (int)(unsigned)total;
            s_first[KS_THREADS] = (int)(total >> 32);
        }
        if (blockIdx.x == 0 && tid < nr) {
            a.row_off[r0 + tid] = (int)(unsigned)exc;
            a.kv_len[r0 + tid] = (int)min((long long)cached + fresh, 0x7FFFFFFFll);
        }
        __syncthreads();
        // the chunk's tokens
        const unsigned stride = gridDim.x * KS_THREADS, first = blockIdx.x * KS_THREADS + tid;
        const unsigned t_end = min((unsigned)total, (unsigned)a.T);
        for (unsigned t = (unsigned)carry + first; t < t_end; t += stride) {
            const int i = search_last(s_row, nr, (int)t);
            const int at = s_cached[i] + ((int)t - s_row[i]);
            const int col = at / a.page, have = pages_of(s_cached[i], a.page);
            int page = -1;
            if (at >= 0 && col < a.cols) {
                const int f = s_first[i] + (col - have);
                if (col < have) page = a.table[(int64_t)(r0 + i) * a.ld_table + col];
                else if (f >= 0 && f < a.n_free) page = a.free_pages[f];
            }
            const long long slot = (long long)page * a.page + (at - col * a.page);
            a.slots[t] = (page >= 0 && slot <= 0x7FFFFFFFll) ? (int)slot : -1;
            a.positions[t] = s_base[i] + at;
        }
        // the chunk's new pages
        const unsigned p_end = (unsigned)(total >> 32);
        for (unsigned f = (unsigned)(carry >> 32) + first; f < p_end;) {
            const int i = search_last(s_first, nr, (int)f);
            const unsigned col = pages_of(s_cached[i], a.page) + (f - s_first[i]);
            if (col < (unsigned)a.cols) {
                a.table[(int64_t)(r0 + i) * a.ld_table + col] = f < (unsigned)a.n_free ? a.free_pages[f] : -1;
                f += stride;
            } else {                   // nor do the request's other pages have a column: on to the next request's
                f += ((unsigned)s_first[i + 1] - f + stride - 1) / stride * stride;
            }
        }
        carry = total;
        __syncthreads();   // the shared arrays are filled again for the next chunk
    }
    // rows that only fill the step up have no slot: whatever writes the cache leaves them out
    for (unsigned t = (unsigned)carry + blockIdx.x * KS_THREADS + tid; t < (unsigned)a.T; t += gridDim.x * KS_THREADS) {
        a.slots[t] = -1;
        a.positions[t] = 0;
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.row_off[a.R] = (int)(unsigned)carry;
        a.taken[0] = (int)(carry >> 32);
    }
}

template <int KS_THREADS>
static cudaError_t launch_kv_slots_n(const KvSlotsArgs& a, int num_sms, cudaStream_t st) {
    const int grid = std::max(1, std::min(num_sms, a.T / KS_THREADS + (a.T % KS_THREADS != 0)));
    return launch_pdl(kv_slots_kernel<KS_THREADS>, dim3(grid), dim3(KS_THREADS), 0, st, a);
}
cudaError_t launch_kv_slots(const KvSlotsArgs& a, int num_sms, cudaStream_t st) {
    return a.R <= 256 ? launch_kv_slots_n<256>(a, num_sms, st) : launch_kv_slots_n<1024>(a, num_sms, st);
}

// ------------------------------------------------------------------------------------------ qk_norm_rope
// Per token t and head h of the queries and keys, with one rounding to bf16 at the end:
//   y     = x * rsqrt(mean(x^2) + eps) * gamma                       (fp32; left out where gamma is null)
//   a_i   = position[axis_i][t] * inv_freq_i                         (in double)
//   (y_i, y_i') -> scale * (y_i cos a_i - y_i' sin a_i, y_i' cos a_i + y_i sin a_i)
// with i' = i + rot/2 (halves) or the pair (2i, 2i+1) (interleaved); channels from rot on are not turned.  Values
// are copied.  Queries go to Q, keys and values to the token's slot of the cache.
//
// Every byte is read and written once, so HBM bounds it from a few hundred tokens on, if enough loads are under way and
// instruction issue stays below.  A head is D/8 lanes of eight channels, a warp takes 32/(D/8) heads at a time (a step) and walks over the
// heads of ONE token, so that the token's cosines and sines are worked out once (two angles per lane, then through shared memory
// into registers) and serve all heads.  A lane's four pairs take four factors each, gamma times cosine or sine, worked out once for the query
// heads and once for the key heads; the norm's factor, known last, multiplies the turned pair.  For rot == D in halves a
// lane holds four channels of each half, so that both members of a pair are in one lane and the rotation needs no shuffle.  The loads of
// four steps are issued together; pointers advance by constants, and the three kinds of heads have loops of their own (with one loop that
// worked out kind, head and addresses for every step it took 150 instructions a step, and 8192 tokens were bound by their issue:
// 44 us, issue slots 64 % used).  With few tokens a token's heads are shared out over several warps instead.
// (Batches of eight, or the whole token on its way into shared memory by one bulk copy with eight warps an SM, were
// slower: 42 and 57 us for 8192 tokens, because the chains of a step want many warps.  Calling a warp's whole part into L2 first changed
// nothing: HBM, reading and writing, is 85 % busy.)
// With fewer heads to a token (32 + 2 x 4, three axes, 5001 tokens: 23.1 us, 0.57 of the issue slots, long scoreboard first among the stalls) the
// chain positions -> angles -> factors in front of the first head's load shows, and key and value steps fill half a batch.
// The angle is reduced in double (position * frequency passes 2^24 for far positions, where fp32 would lose the
// turn entirely) to half turns in [-1, 1], whose sine and cosine are taken in fp32: an error of 2^-23 against a
// rounding step of 2^-8.
constexpr int QR_WARPS = 4;
constexpr int QR_CTAS = 8;      // per SM
constexpr int QR_UNROLL = 4;    // steps whose loads are issued together

struct QkNormRopeArgs {
    const uint16_t* qkv;
    int64_t ld;
    const uint16_t* gamma_q;   // null: no norm
    const uint16_t* gamma_k;
    const float* inv_freq;
    const uint8_t* axis;       // null: axis 0 for every pair
    const int32_t* positions;
    int64_t ld_pos;
    uint16_t* q;
    int64_t ldq;
    uint16_t* k;
    uint16_t* v;
    int64_t page_stride, token_stride, head_stride;
    const int32_t* slots;      // null: token t at slot t
    float eps, scale;
    int T, Hq, Hk, rot, axes, page, n_pages;
    int whole;               // tokens with one warp each; those behind them have warps_per_token
    int warps_per_token;
};

constexpr int ROPE_SPLIT = 0;        // halves, rot == D: a lane holds four channels of each half
constexpr int ROPE_INTERLEAVED = 1;  // pairs (2i, 2i+1)
constexpr int ROPE_PARTIAL = 2;      // halves, rot < D: the partner channel comes by shuffle

template <int D, int MODE>
__global__ void __launch_bounds__(QR_WARPS * 32, MODE == ROPE_SPLIT ? QR_CTAS : QR_CTAS - 2) qk_norm_rope_kernel(const QkNormRopeArgs a) {
    constexpr int LPH = D / 8;       // lanes per head
    constexpr int HPS = 32 / LPH;    // heads per step of a warp
    __shared__ float2 s_cs[QR_WARPS][D / 2];
    grid_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane / LPH, hl = lane % LPH;
    const int nq = (a.Hq + HPS - 1) / HPS, nk = (a.Hk + HPS - 1) / HPS;
    const int steps = nq + 2 * nk;
    const uint32_t job = blockIdx.x * QR_WARPS + warp;      // fewer than 2^31 + QR_WARPS
    const bool shared = job >= (uint32_t)a.whole;
    const uint32_t rest = job - a.whole, w_t = rest / (uint32_t)a.warps_per_token;
    const uint32_t t_u = shared ? a.whole + w_t : job;
    const int part = shared ? (int)(rest - w_t * a.warps_per_token) : 0, parts = shared ? a.warps_per_token : 1;
    grid_dependency_wait();
    if (t_u >= (uint32_t)a.T) return;
    const int t = (int)t_u;
    const int st0 = steps * part / parts, st1 = steps * (part + 1) / parts;
    const uint16_t* row = a.qkv + (int64_t)t * a.ld;
    // first channel of the lane's two groups of four
    const int e0 = MODE == ROPE_SPLIT ? 4 * hl : 8 * hl;
    const int e1 = MODE == ROPE_SPLIT ? D / 2 + 4 * hl : 8 * hl + 4;
    const int half_lanes = a.rot / 16;
    const bool turned = MODE == ROPE_SPLIT || e0 < a.rot;         // rot is a multiple of 16: a lane's eight channels turn together
    const bool upper = MODE == ROPE_PARTIAL && e0 >= a.rot / 2;   // rot / 2 is a multiple of 8
    const int partner = !turned ? lane : upper ? lane - half_lanes : lane + half_lanes;
    const int slot = a.slots ? a.slots[t] : t;

    // cosines and sines of the token; all its positions are fetched beside the pairs' axes
    int pos[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) pos[i] = i < a.axes ? a.positions[(int64_t)i * a.ld_pos + t] : 0;
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
        const int i = k * 32 + lane;
        if (i >= a.rot / 2) break;
        const int ax = a.axis ? min((int)a.axis[i], a.axes - 1) : 0;
        const double ang = (double)(ax == 0 ? pos[0] : ax == 1 ? pos[1] : pos[2]) * (double)a.inv_freq[i];
        double u = ang * 0.31830988618379067154;      // half turns
        u -= 2.0 * rint(u * 0.5);
        float s, c;
        sincospif((float)u, &s, &c);
        s_cs[warp][i] = make_float2(c * a.scale, s * a.scale);
    }
    __syncwarp();
    const int page = slot >= 0 ? slot / a.page : -1;
    const bool cached = slot >= 0 && page < a.n_pages;
    const int64_t cache_row = cached ? (int64_t)page * a.page_stride + (int64_t)(slot - page * a.page) * a.token_stride : 0;

    // Factors of the lane's channels for heads of one kind: SPLIT, INTERLEAVED: y_a = r (x_a ac - x_b bs), y_b = r (x_b bc + x_a as);
    // PARTIAL: y = r x gamma cos + r' x' gamma' (-+ sin), with the partner lane's x' gamma' by shuffle: ac, bc hold gamma, as, bs unused.
    uint64_t ac[2], as[2], bc[2], bs[2];
    float cs[8], sn[8];
    if (MODE == ROPE_PARTIAL) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 v = turned ? s_cs[warp][upper ? e0 + j - a.rot / 2 : e0 + j] : make_float2(1.0f, 0.0f);
            cs[j] = v.x;
            sn[j] = upper ? v.y : -v.y;
        }
    }
    auto factors = [&](const uint16_t* gamma) {
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.0f;
        if (gamma) {
            const uint2 w0 = *reinterpret_cast<const uint2*>(gamma + e0), w1 = *reinterpret_cast<const uint2*>(gamma + e1);
            const uint32_t w[4] = {w0.x, w0.y, w1.x, w1.y};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[2 * j] = __uint_as_float(w[j] << 16);
                g[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            if (MODE == ROPE_PARTIAL) {
                ac[m] = pack2(g[2 * m], g[2 * m + 1]);
                bc[m] = pack2(g[4 + 2 * m], g[5 + 2 * m]);
                as[m] = bs[m] = 0;
                continue;
            }
            const float2 v0 = turned ? s_cs[warp][4 * hl + 2 * m] : make_float2(1.0f, 0.0f);
            const float2 v1 = turned ? s_cs[warp][4 * hl + 2 * m + 1] : make_float2(1.0f, 0.0f);
            const float ga0 = MODE == ROPE_SPLIT ? g[2 * m] : g[4 * m], ga1 = MODE == ROPE_SPLIT ? g[2 * m + 1] : g[4 * m + 2];
            const float gb0 = MODE == ROPE_SPLIT ? g[4 + 2 * m] : g[4 * m + 1], gb1 = MODE == ROPE_SPLIT ? g[5 + 2 * m] : g[4 * m + 3];
            ac[m] = pack2(ga0 * v0.x, ga1 * v1.x);
            as[m] = pack2(ga0 * v0.y, ga1 * v1.y);
            bc[m] = pack2(gb0 * v0.x, gb1 * v1.x);
            bs[m] = pack2(-gb0 * v0.y, -gb1 * v1.y);
        }
    };
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
        // steps of this kind that are the warp's, and how many of them are heads for this lane
        const int H = kind ? a.Hk : a.Hq, first = kind == 0 ? 0 : kind == 1 ? nq : nq + nk;
        const int i0 = max(st0 - first, 0), n = min(st1 - first, kind ? nk : nq) - i0;
        if (n <= 0) continue;
        const int h0 = i0 * HPS + sub, mine = min(n, (H - h0 + HPS - 1) / HPS);
        const uint16_t* src = row + ((kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hk) + h0) * D;
        uint16_t* dst = kind == 0 ? a.q + (int64_t)t * a.ldq + h0 * D : (kind == 1 ? a.k : a.v) + cache_row + (int64_t)h0 * a.head_stride;
        const int64_t dst_step = kind == 0 ? HPS * D : HPS * a.head_stride;
        const int writes = kind == 0 || cached ? mine : 0;
        const uint16_t* gamma = kind == 0 ? a.gamma_q : a.gamma_k;
        if (kind < 2) factors(gamma);
#pragma unroll 1
        for (int b = 0; b < n; b += QR_UNROLL) {
            uint32_t w[QR_UNROLL][4];
#pragma unroll
            for (int j = 0; j < QR_UNROLL; ++j) {
                w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0u;
                if (b + j < mine) {
                    if (MODE == ROPE_SPLIT) {
                        const uint2 x0 = *reinterpret_cast<const uint2*>(src + j * HPS * D + e0), x1 = *reinterpret_cast<const uint2*>(src + j * HPS * D + e1);
                        w[j][0] = x0.x; w[j][1] = x0.y; w[j][2] = x1.x; w[j][3] = x1.y;
                    } else {
                        const uint4 x0 = *reinterpret_cast<const uint4*>(src + j * HPS * D + e0);
                        w[j][0] = x0.x; w[j][1] = x0.y; w[j][2] = x0.z; w[j][3] = x0.w;
                    }
                }
            }
            src += QR_UNROLL * HPS * D;
            // Four independent chains (sum of squares, shuffles, rsqrt, rotation) side by side: no branch between them, so the last batch
            // may turn heads that are not there.
            if (kind < 2) {
#pragma unroll
                for (int j = 0; j < QR_UNROLL; ++j) {
                    uint64_t x[4];           // SPLIT: (a0 a1) (a2 a3) (b0 b1) (b2 b3); INTERLEAVED, PARTIAL: channels in order
#pragma unroll
                    for (int m = 0; m < 4; ++m) x[m] = pack2(__uint_as_float(w[j][m] << 16), __uint_as_float(w[j][m] & 0xFFFF0000u));
                    float r = 1.0f;
                    if (gamma) {
                        float s0, s1;
                        unpack2(add2(fma2(x[0], x[0], mul2(x[1], x[1])), fma2(x[2], x[2], mul2(x[3], x[3]))), s0, s1);
                        float ss = s0 + s1;
#pragma unroll
                        for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
                        r = rsqrtf(ss * (1.0f / D) + a.eps);
                    }
                    const uint64_t r2 = pack2(r, r);
                    if (MODE == ROPE_PARTIAL) {
                        float v[8], y[8];
                        unpack2(mul2(x[0], mul2(ac[0], r2)), v[0], v[1]);
                        unpack2(mul2(x[1], mul2(ac[1], r2)), v[2], v[3]);
                        unpack2(mul2(x[2], mul2(bc[0], r2)), v[4], v[5]);
                        unpack2(mul2(x[3], mul2(bc[1], r2)), v[6], v[7]);
#pragma unroll
                        for (int m = 0; m < 8; ++m) {
                            const float o = __shfl_sync(0xFFFFFFFFu, v[m], partner);
                            y[m] = turned ? v[m] * cs[m] + o * sn[m] : v[m];
                        }
#pragma unroll
                        for (int m = 0; m < 4; ++m) w[j][m] = bf162_bits(__floats2bfloat162_rn(y[2 * m], y[2 * m + 1]));
                    } else {
                        uint64_t xa[2] = {x[0], x[1]}, xb[2] = {x[2], x[3]};
                        if (MODE == ROPE_INTERLEAVED) {
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                float p, q, u, z;
                                unpack2(x[2 * m], p, q);
                                unpack2(x[2 * m + 1], u, z);
                                xa[m] = pack2(p, u);
                                xb[m] = pack2(q, z);
                            }
                        }
                        float ya[4], yb[4];
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            unpack2(mul2(r2, fma2(xa[m], ac[m], mul2(xb[m], bs[m]))), ya[2 * m], ya[2 * m + 1]);
                            unpack2(mul2(r2, fma2(xb[m], bc[m], mul2(xa[m], as[m]))), yb[2 * m], yb[2 * m + 1]);
                        }
#pragma unroll
                        for (int m = 0; m < 4; ++m)
                            w[j][m] = MODE == ROPE_SPLIT ? bf162_bits(m < 2 ? __floats2bfloat162_rn(ya[2 * m], ya[2 * m + 1])
                                                                            : __floats2bfloat162_rn(yb[2 * m - 4], yb[2 * m - 3]))
                                                         : bf162_bits(__floats2bfloat162_rn(ya[m], yb[m]));
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < QR_UNROLL; ++j) {
                if (b + j < writes) {
                    if (MODE == ROPE_SPLIT) {
                        *reinterpret_cast<uint2*>(dst + e0) = make_uint2(w[j][0], w[j][1]);
                        *reinterpret_cast<uint2*>(dst + e1) = make_uint2(w[j][2], w[j][3]);
                    } else {
                        *reinterpret_cast<uint4*>(dst + e0) = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
                    }
                }
                dst += dst_step;
            }
        }
    }
}

template <int D, int MODE>
static cudaError_t launch_qk_norm_rope_mode(QkNormRopeArgs a, int num_sms, cudaStream_t st) {
    const int hps = 32 / (D / 8);
    const int steps = (a.Hq + hps - 1) / hps + 2 * ((a.Hk + hps - 1) / hps);
    // A warp per token for as many rounds of the machine's resident warps as are full.  The tokens behind them (all, where there are few) are spread
    // over more warps while those fill half of the machine: the last round is then as short as its work.  From CUDA graphs on three inputs
    // in turn, 32 + 2 x 8 heads of 128: 5001 tokens (1.06 rounds) 26.7 us like this; all of them in 1 / 2 / 4 / 8 warps each 30.8 / 28.6 / 32.8 /
    // 43.1, because every warp works out the angles again; 8192 tokens (1.73 rounds) 37.4 like this, 37.4 / 39.0 / 47.7 / 67.5; 256 tokens
    // 6.2 like this, 10.3 / 6.2 / 6.2 / 6.2.
    const int resident = num_sms * QR_WARPS * (MODE == ROPE_SPLIT ? QR_CTAS : QR_CTAS - 2);
    a.whole = a.T / resident * resident;
    const int rest = a.T - a.whole;
    a.warps_per_token = rest ? std::max(1, std::min(resident / 2 / rest, std::min(steps, 32))) : 1;
    const int64_t jobs = (int64_t)a.whole + (int64_t)rest * a.warps_per_token;
    return launch_pdl(qk_norm_rope_kernel<D, MODE>, dim3((unsigned)((jobs + QR_WARPS - 1) / QR_WARPS)), dim3(QR_WARPS * 32), 0, st, a);
}

template <int D>
static cudaError_t launch_qk_norm_rope_d(const QkNormRopeArgs& a, bool interleaved, int num_sms, cudaStream_t st) {
    if (interleaved) return launch_qk_norm_rope_mode<D, ROPE_INTERLEAVED>(a, num_sms, st);
    if (a.rot == D) return launch_qk_norm_rope_mode<D, ROPE_SPLIT>(a, num_sms, st);
    return launch_qk_norm_rope_mode<D, ROPE_PARTIAL>(a, num_sms, st);
}

cudaError_t launch_qk_norm_rope(const QkNormRopeArgs& a, int D, bool interleaved, int num_sms, cudaStream_t st) {
    return D == 128 ? launch_qk_norm_rope_d<128>(a, interleaved, num_sms, st) : launch_qk_norm_rope_d<64>(a, interleaved, num_sms, st);
}

}  // namespace osc
