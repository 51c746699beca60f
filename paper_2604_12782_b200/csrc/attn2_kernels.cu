// Attention for segments with many rows per key/value head (a prefix under many requests, a piece of a prompt):
// tcgen05 kernel on the tile line of attn_kernels.cu.
//
// A unit is two tiles of up to 128 rows (tokens x query heads of one key/value head).  S = Q K^T and O += P V
// both run on the fifth-generation tensor cores: Q, K and V tiles come by TMA into shared memory, S, P and O live in TMEM (P, the weights
// in bf16, is read from there as the A operand).  Two streams run in counterphase, each with its own P, O and warpgroup (one
// row per thread): while one stream's softmax runs, the other's products do.
//   both row tiles filled: stream s is row tile s; they share every K and V tile.
//   one row tile:          both streams take the same rows and every other key tile; the results are joined
//                          at the end of the unit (a thread can read both O rows: they lie in its lanes).
// With D = 128 two S (128 x 128), two P and two O do not fit TMEM.  The streams share ONE S: a softmax thread takes its whole row of scores
// into registers at once, and the other stream's product can go there a few hundred cycles later.  (Each stream with its own S and P in the
// columns of that S made a stream's steps run strictly one after the other - S, softmax, P V, next S: 3700 cycles for 128 keys of both tiles,
// tensor pipe 47 % busy; own S and P with 64-key tiles: 5500, twice the MMA warp's steps, whose overhead was then what counted.)
//
//   warps 0-3, 4-7 : softmax of stream 0, 1, and their epilogue
//   warp 8         : TMA (a key tile is loaded page by page; a page that is not there reads as zeros)
//   warps 9, 11    : MMA issue of S, of P V (warp 9 owns TMEM)
//   warp 10        : the units of the CTA's share, for everyone else
//
// Bound by the tensor pipe and the exponentials alike (72 % of the cycles each): 2560 cycles per 128 keys of both tiles, of which the four
// products are 2080 and the exponentials 2048, and 7000 cycles to end a unit and begin the next one (5000 of them the epilogue; a second Q and a second pair of O
// to hide it behind have no room).  8001 tokens of prompts behind 2048 keys: 375 us from the plan's end on, 1.33 PFLOP/s, replayed from a graph in a short
// run (402 cold, under the profiler); the power limit takes a sixth of that in a loop of seconds.
//
// P V with the weights of the running maximum as it stands: O is rescaled in TMEM only when the maximum has moved by
// more than 2^8 (see AT_SLACK), by the softmax threads themselves, between the P V before and the one to come.
#include <algorithm>

#include "common.cuh"

namespace osc {

struct AttnWideArgs {
    CUtensorMap tm_q;     // [T][Hq][D], box 64 channels x G heads x whole tokens of a tile
    CUtensorMap tm_k;     // [n_pages][Hk][page][D], box 64 channels x min(page, 128) tokens of one head
    CUtensorMap tm_v;
    AttnArgs a;
};

constexpr int AW_SOFTMAX_WARPS = 8;
constexpr int AW_THREADS = (AW_SOFTMAX_WARPS + 4) * 32;
// Registers: launched with 168 a thread (12 warps).  The softmax warpgroups hold a row of 128 scores each thread and take
// 208, the last one gives down to 80.
constexpr int AW_REGS_LAUNCH = 168, AW_REGS_SOFTMAX = 208, AW_REGS_OTHER = 80;
static_assert(AW_SOFTMAX_WARPS * AW_REGS_SOFTMAX + 4 * AW_REGS_OTHER <= (AW_SOFTMAX_WARPS + 4) * AW_REGS_LAUNCH, "register split");
template <int R>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D>
struct WideCfg {
    static constexpr int HALVES = D / 64;                        // 128-byte swizzle rows hold 64 channels
    static constexpr int QHALF_BYTES = 128 * 128;                // 128 rows of 64 channels
    static constexpr int QTILE_BYTES = HALVES * QHALF_BYTES;
    static constexpr int HALF_BYTES = AT_WIDE_KEYS * 128;        // 128 keys of 64 channels
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;
    static constexpr int STAGES = D == 128 ? 2 : 4;              // K tiles, and as many V tiles
    static constexpr int OUT_BYTES = AW_SOFTMAX_WARPS * 2048;    // every softmax warp's 32 rows x 64 bytes of O on the way out
    static constexpr int ROW_FLOATS = 2 * 2 * 2 * 128;           // [parity][stream][128] maxima and sums of a unit
    static constexpr int BAR_BYTES = 320;
    static constexpr int SMEM = 2 * QTILE_BYTES + 2 * STAGES * TILE_BYTES + OUT_BYTES + ROW_FLOATS * 4 + BAR_BYTES + 2 * 64 + 1024;
    static constexpr int TM_S = 0;         // TMEM columns: S (128), P0, P1 (64 each), O0, O1 (D each)
    static constexpr int TM_P = 128;
    static constexpr int TM_O = 256;
    static_assert(SMEM <= 232448, "shared memory");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int x, int y, int z, int w) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// D[tmem] (+)= A[tmem, 16-bit pairs] . B[smem]
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                 "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Descriptor of a V tile as the B operand of P V: B is [channel][key], stored with the channels contiguous (64 to a
// swizzled 128-byte row).  Along channels the next 64 are HALF_BYTES away (leading offset), along keys the next 8
// are 1024 bytes away (stride offset).
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t saddr, uint32_t half_bytes) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFF) >> 4);
    d |= static_cast<uint64_t>(half_bytes >> 4) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
constexpr uint32_t IDESC_B_MN = 1u << 16;   // B operand with its N extent contiguous

// What the roles need to know of a unit, or of the part of it that the CTA's share has: key tiles [ka, ka + n).  The units
// warp walks over the line and keeps two of these ahead in shared memory.
struct __align__(16) WideUnit {
    int ka, n;          // n = 0: the share is done
    int cnt[2];         // key tiles of stream 0 and 1
    int pair;           // both row tiles filled: stream s has row tile s and all its key tiles; else every other key tile
    int nf;             // key tiles in front (the group's prefix), before the own keys'
    int plen, klen;     // keys in front, own keys
    int front, seg;     // segments that name the pages of the keys in front and of the own keys
    int h, row0;        // head, first row of the unit (token index in Q)
    int tok0, tokens;   // first token of the unit and number of tokens, inside the segment
    int causal;
    int out;            // bits: OUT_*
};
constexpr int OUT_SPLIT = 1, OUT_TWO = 2, OUT_OWN = 4, OUT_LATER = 8;   // OUT_LATER: the share has tiles before this unit

// keys of key tile kt before any mask
__device__ __forceinline__ int unit_left(const WideUnit& w, int kt) {
    return kt < w.nf ? w.plen - kt * AT_WIDE_KEYS : w.klen - (kt - w.nf) * AT_WIDE_KEYS;
}

template <int D>
__global__ void __launch_bounds__(AW_THREADS, 1) attn_wide_kernel(const __grid_constant__ AttnWideArgs args) {
    using C = WideCfg<D>;
    constexpr int STAGES = C::STAGES, NSW = AW_SOFTMAX_WARPS;
    const AttnArgs& a = args.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring = smem + 2 * C::QTILE_BYTES;
    uint8_t* out_tiles = ring + 2 * STAGES * C::TILE_BYTES;
    float2* unit_ml = reinterpret_cast<float2*>(out_tiles + C::OUT_BYTES);  // [parity][stream][128]
    uint64_t* bars = reinterpret_cast<uint64_t*>(unit_ml + 4 * 128);
    uint64_t* full = bars;               // [2][STAGES]: K, V
    uint64_t* empty = bars + 2 * STAGES; // [2][STAGES]
    uint64_t* q_full = bars + 4 * STAGES;
    uint64_t* q_empty = q_full + 1;
    uint64_t* s_full = q_full + 2;       // [2]
    uint64_t* p_full = q_full + 4;       // [2]
    uint64_t* pv_done = q_full + 6;      // [2]
    uint64_t* u_full = q_full + 8;       // [2]
    uint64_t* u_empty = q_full + 10;     // [2]
    uint64_t* s_empty = q_full + 12;
    uint64_t* o_empty = q_full + 13;
    uint64_t* e_full = q_full + 14;
    uint64_t* drain_bar = q_full + 15;
    constexpr int BARS = 4 * STAGES + 16;
    WideUnit* units = reinterpret_cast<WideUnit*>(reinterpret_cast<uint8_t*>(bars) + C::BAR_BYTES);   // [2]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    static_assert(BARS * 8 + 8 <= C::BAR_BYTES, "barriers");

    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < BARS; ++i) {
            const int b = i - 4 * STAGES;      // all barriers take one arrival but these
            mbar_init(&bars[i], b == 4 || b == 5 || b == 12 ? NSW / 2 : b == 10 || b == 11 ? NSW + 3 : b == 13 || b == 14 ? NSW : b == 15 ? 2 : 1);
        }
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&args.tm_q);
        prefetch_tmap(&args.tm_k);
        prefetch_tmap(&args.tm_v);
    }
    if (warp == NSW + 1) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
    grid_dependency_wait();
    grid_launch_dependents();   // not before: the few-row kernel counts on the plan being there when it begins
    const int tpt = a.tpt;
    const uint32_t ring0 = smem_u32(ring);

    if (warp >= NSW) {
        regs_dec<AW_REGS_OTHER>();
        if (warp == NSW + 2) {
            // ------------------------------------------------------------------------------------- units
            const int S = a.P + a.R;
            const int N = a.plan.wide_start[S], q = a.plan.share[1];
            const int x0 = (int)min((int64_t)q * blockIdx.x, (int64_t)N), x1 = (int)min((int64_t)x0 + q, (int64_t)N);
            Cursor<WideUnits> cur;
            const LineSource<false> src = {a.plan.seg, a.plan.wide_start};
            if (lane == 0) a.plan.cut[1][blockIdx.x].tiles = 0;
            int b = 0, x = x0;
            uint32_t ph = 0;
            if (x0 < x1) {
                cur.seek(a, src, S, x0);
                if (cur.kt < 0) { x -= cur.kt; cur.kt = 0; }         // in front of the unit's tiles
            }
            while (true) {
                WideUnit w = {};
                if (x < x1) {
                    w.ka = cur.kt;
                    w.n = min(cur.nt - cur.kt, x1 - x);
                    w.tok0 = cur.u * 2 * tpt;
                    w.tokens = min(cur.g.n - w.tok0, 2 * tpt);
                    w.pair = w.tokens > tpt;
                    w.nf = front_tiles<WideUnits>(a, cur.g);
                    if (w.pair) {
                        const int nt0 = w.nf + (seg_sees(cur.g, w.tok0 + tpt - 1) + AT_WIDE_KEYS - 1) / AT_WIDE_KEYS;
                        w.cnt[0] = max(min(w.ka + w.n, nt0) - w.ka, 0);
                        w.cnt[1] = w.n;
                    } else {
                        w.cnt[0] = (w.n + 1) / 2;
                        w.cnt[1] = w.n / 2;
                    }
                    w.plen = cur.g.plen;
                    w.klen = cur.g.klen;
                    w.front = cur.g.group;
                    w.seg = cur.s;
                    w.h = cur.h;
                    w.row0 = cur.g.t0 + w.tok0;
                    w.causal = cur.g.flags & SEG_OWN ? cur.g.n : 0;
                    w.out = (w.n < cur.nt ? OUT_SPLIT : 0) | (cur.g.flags & SEG_TWO ? OUT_TWO : 0) | (cur.s >= a.P ? OUT_OWN : 0) | (x > x0 ? OUT_LATER : 0);
                }
                if (!wait_bounded(&u_empty[b], ph ^ 1u, abort_flag, 76)) break;
                if (lane == 0) {
                    units[b] = w;
                    mbar_arrive(&u_full[b]);
                }
                if (++b == 2) { b = 0; ph ^= 1u; }
                if (w.n == 0) break;
                if (x + w.n == x1 && lane == 0)
                    tell_cut(a.plan.cut[1] + blockIdx.x, x - w.ka, x - w.ka + cur.nt, x0, x1, q, cur.h, cur.u, cur.g);
                x += w.n;
                if (x < x1) {
                    cur.next_unit(a, src, SEG_WIDE);
                    x += WideUnits::LEAD;
                }
            }
        } else if (warp == NSW) {
            // --------------------------------------------------------------------------------------- TMA
            const int bt = min(1 << a.page_shift, AT_WIDE_KEYS);     // tokens of a box
            const int boxes = AT_WIDE_KEYS / bt * C::HALVES;         // of a K or V tile: at most 16, one lane each
            const int mine = lane / C::HALVES, half = lane % C::HALVES;
            uint32_t n_k = 0, n_v = 0;      // K and V loads so far: tile n in slot n % STAGES, phase n / STAGES
            int b = 0;
            uint32_t q_ph = 0, u_ph = 0;
            while (true) {
                if (!wait_bounded(&u_full[b], u_ph, abort_flag, 60)) goto stop_loads;
                const WideUnit& w = units[b];
                const int ka = w.ka, n = w.n, nf = w.nf, h = w.h;
                if (n == 0) break;
                const int32_t* own_pages = seg_pages(a, w.seg);
                const int32_t* front_pages = nf ? seg_pages(a, w.front) : own_pages;
                int page = 0, place = 0;
                // K one tile ahead of V: a K slot is free again long before the V slot of the same tile
                for (int i = 0; i <= n; ++i) {
                    const int v_page = page, v_place = place;
                    if (i < n) {
                        const int kt = ka + i;
                        page = a.n_pages;      // a box past the last page is filled with zeros
                        place = 0;
                        if (lane < boxes) {
                            const int key = (kt < nf ? kt : kt - nf) * AT_WIDE_KEYS + mine * bt;
                            if (mine * bt < unit_left(w, kt)) {          // a length is within the list's columns
                                const int p = (kt < nf ? front_pages : own_pages)[key >> a.page_shift];
                                if (p >= 0 && p < a.n_pages) page = p;
                                place = key & ((1 << a.page_shift) - 1);
                            }
                        }
                    }
#pragma unroll 1
                    for (int v = 0; v < 2; ++v) {
                        if (v ? i == 0 : i == n) continue;
                        const uint32_t t = v ? n_v : n_k, st = v * STAGES + t % STAGES;
                        if (!wait_bounded(&empty[st], (t / STAGES + 1) & 1u, abort_flag, 62)) goto stop_loads;
                        if (lane == 0) mbar_arrive_expect_tx(&full[st], C::TILE_BYTES);
                        __syncwarp();
                        if (lane < boxes)
                            tma_load_4d(ring0 + st * C::TILE_BYTES + half * C::HALF_BYTES + mine * bt * 128, v ? &args.tm_v : &args.tm_k, &full[st],
                                        half * 64, v ? v_place : place, h, v ? v_page : page);
                        if (v) ++n_v; else ++n_k;
                    }
                    if (i == 0) {      // behind the first K: Q, whose place is free when the unit before has no more S to come
                        if (!wait_bounded(q_empty, q_ph ^ 1u, abort_flag, 61)) goto stop_loads;
                        q_ph ^= 1u;
                        const int tiles = w.pair ? 2 : 1;
                        if (lane == 0) mbar_arrive_expect_tx(q_full, (uint32_t)(tiles * C::HALVES * tpt * a.G * 128));
                        __syncwarp();
                        if (lane < tiles * C::HALVES)
                            tma_load_3d(smem_u32(smem + mine * C::QTILE_BYTES + half * C::QHALF_BYTES), &args.tm_q, q_full, half * 64, h * a.G,
                                        w.row0 + mine * tpt);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&u_empty[b]);
                if (++b == 2) { b = 0; u_ph ^= 1u; }
            }
        stop_loads:
            __syncwarp();
            if (*abort_flag) {      // gave up somewhere: the copies under way land before the CTA's memory goes away
                int dummy = 0;
                volatile int* never = &dummy;
                for (int v = 0; v < 2; ++v) {
                    const uint32_t t = v ? n_v : n_k;
                    for (uint32_t i = t > STAGES ? t - STAGES : 0; i < t; ++i) wait_bounded(&full[v * STAGES + i % STAGES], (i / STAGES) & 1u, never, 63);
                }
                wait_bounded(q_full, q_ph ^ 1u, never, 64);
            }
        } else {
            // --------------------------------------------------------------------------------- MMA: S, and P V
            // Two warps, because the products are independent of each other (S and P have columns of their own) and an issuing warp is
            // held up until its MMAs are nearly through: with one warp for all four products of a step, its waits and address
            // arithmetic (370 cycles each) came on top of the 520 cycles of each product.
            // The whole warp walks through the loops (one elected lane issues), and what it reads from shared memory goes through a shuffle:
            // only then do the descriptors stay in uniform registers.
            auto uni = [](int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); };
            const bool s_warp = warp == NSW + 1;
            const uint64_t q_desc = smem_desc_sw128(smem_u32(smem)), k_desc = smem_desc_sw128(ring0);
            const uint64_t v_desc = smem_desc_sw128_mn(ring0, C::HALVES > 1 ? C::HALF_BYTES : 1024);
            constexpr uint32_t IDESC_S = idesc_bf16(128, AT_WIDE_KEYS), IDESC_O = idesc_bf16(128, D) | IDESC_B_MN;
            uint32_t base = 0;                 // tiles of the units before
            uint32_t q_ph = 0, p_ph = 0, se_ph = 1, oe_ph = 1, u_ph = 0;
            int b = 0;
            while (true) {
                if (!wait_bounded(&u_full[b], u_ph, abort_flag, 78)) goto done;
                const WideUnit& w = units[b];
                const int n = uni(w.n), cnt0 = uni(w.cnt[0]), cnt1 = uni(w.cnt[1]), pair = uni(w.pair), most = max(cnt0, cnt1);
                if (n == 0) break;
                if (s_warp) {
                    if (!wait_bounded(q_full, q_ph, abort_flag, 65)) goto done;
                    q_ph ^= 1u;
                    for (int j = 0; j < most; ++j) {
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            if (j >= (s ? cnt1 : cnt0)) continue;
                            const uint32_t t = base + (pair ? j : 2 * j + s), stg = t % STAGES;
                            if (!wait_bounded(&full[stg], (t / STAGES) & 1u, abort_flag, 66)) goto done;
                            if (!wait_bounded(s_empty, se_ph, abort_flag, 84)) goto done;     // the S before has been read
                            se_ph ^= 1u;
                            tc_fence_after();
                            const uint64_t qd = q_desc + (pair ? s * (C::QTILE_BYTES >> 4) : 0), kd = k_desc + stg * (C::TILE_BYTES >> 4);
                            if (elect_one()) {
#pragma unroll
                                for (int k = 0; k < D / 16; ++k)
                                    mma_f16(tmem + C::TM_S, qd + (((k / 4) * C::QHALF_BYTES + (k % 4) * 32) >> 4),
                                            kd + (((k / 4) * C::HALF_BYTES + (k % 4) * 32) >> 4), IDESC_S, k ? 1u : 0u);
                                tc_commit(&s_full[s]);
                                if (!pair || s == 1) tc_commit(&empty[stg]);
                            }
                            __syncwarp();
                        }
                    }
                    if (elect_one()) tc_commit(q_empty);      // no more S of this unit
                    __syncwarp();
                } else {
                    // tiles of the unit's part that end inside, counted from its first
                    const int ka = uni(w.ka), nf = uni(w.nf), plen = uni(w.plen), klen = uni(w.klen);
                    const int end_front = plen % AT_WIDE_KEYS ? nf - 1 - ka : -1, end_own = klen % AT_WIDE_KEYS ? nf + klen / AT_WIDE_KEYS - ka : -1;
                    if (!wait_bounded(o_empty, oe_ph, abort_flag, 67)) goto done;      // the epilogue of the unit before has read O
                    oe_ph ^= 1u;
                    for (int i = 0; i < most; ++i) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            if (i >= (x ? cnt1 : cnt0)) continue;
                            const int tile = pair ? i : 2 * i + x;
                            const uint32_t t = base + tile, stg = STAGES + t % STAGES;
                            if (!wait_bounded(&full[stg], (t / STAGES) & 1u, abort_flag, 68)) goto done;
                            if ((tile == end_front || tile == end_own) && (x == 0 || !pair || i >= cnt0)) {
                                // Behind the last key of a list the page holds whatever was there before: a NaN or Inf would survive its weight of 0.
                                const int left = unit_left(w, ka + tile);
                                uint8_t* v = smem + 2 * C::QTILE_BYTES + stg * C::TILE_BYTES;
                                for (int c = left * 8 + lane; c < AT_WIDE_KEYS * 8; c += 32)
                                    for (int hf = 0; hf < C::HALVES; ++hf)
                                        *reinterpret_cast<uint4*>(v + hf * C::HALF_BYTES + c * 16) = make_uint4(0u, 0u, 0u, 0u);
                                fence_proxy_async_smem();
                                __syncwarp();
                            }
                            if (!wait_bounded(&p_full[x], (p_ph >> x) & 1u, abort_flag, 69)) goto done;
                            p_ph ^= 1u << x;
                            tc_fence_after();
                            const uint64_t vd = v_desc + stg * (C::TILE_BYTES >> 4);
                            if (elect_one()) {
#pragma unroll
                                for (int k = 0; k < AT_WIDE_KEYS / 16; ++k)
                                    mma_f16_ts(tmem + C::TM_O + x * D, tmem + C::TM_P + x * (AT_WIDE_KEYS / 2) + k * 8, vd + k * 128, IDESC_O,
                                               (i | k) ? 1u : 0u);
                                tc_commit(&pv_done[x]);
                                if (!pair || x == 1) tc_commit(&empty[stg]);
                            }
                            __syncwarp();
                        }
                    }
                }
                base += n;
                if (lane == 0) mbar_arrive(&u_empty[b]);
                if (++b == 2) { b = 0; u_ph ^= 1u; }
            }
        }
    } else {
        // ------------------------------------------------------------------------------------------ softmax
        regs_inc<AW_REGS_SOFTMAX>();
        const int s = warp >> 2;                                         // stream
        const int r = threadIdx.x & 127;                                 // row of the tile = TMEM lane
        const int my_tok = r * a.inv_g >> 16;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + C::TM_S, t_p = tmem + lanes + C::TM_P + s * (AT_WIDE_KEYS / 2), t_o = tmem + lanes + C::TM_O;
        const float scale = a.scale_log2;
        uint32_t s_ph = 0, pv_ph = 0, e_ph = 0, u_ph = 0;
        int b = 0;
        while (true) {
            if (!wait_bounded(&u_full[b], u_ph, abort_flag, 79)) goto done;
            const WideUnit& w = units[b];
            if (w.n == 0) break;
            float m = -INFINITY, l = 0.0f;
            const int cnt = w.cnt[s];
            {
                const int tok = (w.pair ? s * tpt : 0) + my_tok;         // token inside the unit
                const bool valid = my_tok < tpt && tok < w.tokens;
                const int nf = w.nf, step = w.pair ? 1 : 2;
                // own keys that the row sees; a row that is not there sees all
                const int sees = valid && w.causal ? max(w.klen - w.causal + w.tok0 + tok + 1, 0) : w.klen;
                int kt = w.pair ? w.ka : w.ka + s;
                for (int i = 0; i < cnt; ++i, kt += step) {
                    if (!wait_bounded(&s_full[s], s_ph, abort_flag, 70)) goto done;
                    s_ph ^= 1u;
                    tc_fence_after();
                    uint32_t v[4][32];
#pragma unroll
                    for (int j = 0; j < 4; ++j) tmem_ld_32x32(t_s + j * 32, v[j]);
                    const int left = kt < nf ? w.plen - kt * AT_WIDE_KEYS : sees - (kt - nf) * AT_WIDE_KEYS;      // keys of the tile that the row sees
                    const bool whole = __all_sync(0xFFFFFFFFu, left >= AT_WIDE_KEYS);
                    tmem_ld_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_empty);
                    if (!whole) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (j * 32 + e >= left) v[j][e] = 0xFF800000u;
                    }
                    float mx[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mx[j] = __uint_as_float(v[j][0]);
#pragma unroll
                        for (int e = 1; e < 31; e += 2) mx[j] = max3(mx[j], __uint_as_float(v[j][e]), __uint_as_float(v[j][e + 1]));
                        mx[j] = fmaxf(mx[j], __uint_as_float(v[j][31]));
                    }
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                    const bool move = top > m + AT_SLACK;
                    const float f = move ? exp2_approx(m - top) : 1.0f;
                    if (move) m = top;
                    const float ref = m == -INFINITY ? 0.0f : -m;
                    const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(ref, ref);
                    uint64_t sum[2] = {0, 0};
                    uint32_t pk[4][16];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float p0, p1;
                            unpack2(fma2(pack2(__uint_as_float(v[j][e]), __uint_as_float(v[j][e + 1])), scale2, ref2), p0, p1);
                            p0 = exp2_approx(p0);
                            p1 = exp2_approx(p1);
                            sum[(e / 2) & 1] = add2(sum[(e / 2) & 1], pack2(p0, p1));
                            pk[j][e / 2] = bf162_bits(__floats2bfloat162_rn(p0, p1));      // bf16 as V is: operands of one type
                        }
                    if (i > 0) {      // the P V before has read P, and O is not being written
                        if (!wait_bounded(&pv_done[s], pv_ph, abort_flag, 82)) goto done;
                        pv_ph ^= 1u;
                        if (__any_sync(0xFFFFFFFFu, move)) {
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld_x16(t_o + s * D + c, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st_32x16(t_o + s * D + c, o);
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) tmem_st_32x16(t_p + j * 16, pk[j]);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[s]);
                    float s0, s1;
                    unpack2(add2(sum[0], sum[1]), s0, s1);
                    l = l * f + (s0 + s1);
                }
            }
            // ---- the unit's rows: into O, or as (m, l, O) into the workspace
            const bool pair = w.pair, have0 = w.cnt[0] > 0, have1 = w.cnt[1] > 0;
            if (cnt > 0) {
                if (!wait_bounded(&pv_done[s], pv_ph, abort_flag, 71)) goto done;
                pv_ph ^= 1u;
            }
            // both row tiles filled: a stream's own rows; else the two warpgroups share out the columns of the one tile, O being the two
            // streams' joined
            const int first = pair ? s : 0;
            const bool joined = !pair && have1, have = first ? have1 : have0;
            float m1 = -INFINITY, l1 = 0.0f;
            if (!pair) {
                float2* ml = unit_ml + (e_ph & 1) * 256;
                ml[s * 128 + r] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(e_full);
                if (!wait_bounded(e_full, e_ph & 1, abort_flag, 83)) goto done;
                e_ph ^= 1u;
                m = ml[r].x;
                l = ml[r].y;
                m1 = ml[128 + r].x;
                l1 = ml[128 + r].y;
            }
            tc_fence_after();
            float c0 = m == -INFINITY ? 0.0f : 1.0f, c1 = 0.0f;
            if (joined) {
                const float mn = fmaxf(m, m1);
                c0 = mn == -INFINITY ? 0.0f : exp2_approx(m - mn);
                c1 = mn == -INFINITY ? 0.0f : exp2_approx(m1 - mn);
                m = mn;
                l = l * c0 + l1 * c1;
            }
            const int out = w.out, tok0 = pair ? s * tpt : 0, tokens = w.tokens, hq0 = w.h * a.G, row0 = w.row0;
            const bool direct = !(out & (OUT_SPLIT | OUT_TWO));
            if (direct) {
                const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
                c0 *= inv;
                c1 *= inv;
            }
            const int slot0 = AT_FEW_SLOTS + (blockIdx.x * 2 + (out & OUT_LATER ? 1 : 0)) * (2 * AT_WIDE_TILE) + (pair ? s * AT_WIDE_TILE : 0);
            // token and head of tile row x; whether there is one
            auto row_of = [&](int x, int& tok, int& hq) -> bool {
                const int t = x * a.inv_g >> 16;
                tok = row0 + tok0 + t;
                hq = hq0 + x - t * a.G;
                return t < tpt && tok0 + t < tokens;
            };
            // its row of the partial results
            auto part_row = [&](int x, int tok, int hq) -> int { return out & OUT_SPLIT ? slot0 + x : dense_row(a, out & OUT_OWN ? 1 : 0, tok * a.Hq + hq); };
            if (pair || s == 0) {
                int tok, hq;
                if (row_of(r, tok, hq)) {
                    if (!direct) a.ml[part_row(r, tok, hq)] = piece_ml(m, l);
                    else if (a.lse) a.lse[tok * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
                }
            }
            // A thread holds a row; through shared memory (16-byte units swizzled by the row) four lanes write 64 bytes of one row side by side,
            // eight rows at a time: 32 channels in bf16, or 16 of a partial result.  (Written by the rows' own threads, 16 bytes of 32 rows in one
            // store, a unit took 7000 to 10000 cycles to get out; 16 channels at a time for bf16 too, and with two divisions a row, 8200.)
            int64_t to[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int x = (warp & 3) * 32 + y * 8 + lane / 4;
                int tok, hq;
                to[y] = !row_of(x, tok, hq) ? -1 : direct ? tok * a.ldo + hq * D : (int64_t)part_row(x, tok, hq) * D;
            }
            uint8_t* tile = out_tiles + warp * 2048;
            const int cols = pair ? D : D / 2, col0 = pair ? 0 : s * cols;
            const int e = lane & 3, wsw = (lane >> 1) & 3, rsw = (lane >> 3) & 3;
            if (direct) {
#pragma unroll 1
                for (int c = col0; c < col0 + cols; c += 32) {
                    uint32_t x[32], pk[16];
#pragma unroll
                    for (int y = 0; y < 32; ++y) x[y] = 0u;
                    if (have) {
                        tmem_ld_32x32(t_o + first * D + c, x);
                        tmem_ld_wait();
                    }
                    float o[32];
#pragma unroll
                    for (int y = 0; y < 32; ++y) o[y] = c0 != 0.0f ? __uint_as_float(x[y]) * c0 : 0.0f;
                    if (joined) {
                        tmem_ld_32x32(t_o + D + c, x);
                        tmem_ld_wait();
                        if (c1 != 0.0f) {
#pragma unroll
                            for (int y = 0; y < 32; ++y) o[y] = fmaf(__uint_as_float(x[y]), c1, o[y]);
                        }
                    }
#pragma unroll
                    for (int y = 0; y < 16; ++y) pk[y] = bf162_bits(__floats2bfloat162_rn(o[2 * y], o[2 * y + 1]));
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        *reinterpret_cast<uint4*>(tile + lane * 64 + ((y ^ wsw) * 16)) = make_uint4(pk[4 * y], pk[4 * y + 1], pk[4 * y + 2], pk[4 * y + 3]);
                    __syncwarp();
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint4 q = *reinterpret_cast<const uint4*>(tile + (y * 8 + lane / 4) * 64 + ((e ^ rsw) * 16));
                        if (to[y] >= 0) *reinterpret_cast<uint4*>(a.o + to[y] + c + e * 8) = q;
                    }
                    __syncwarp();
                }
            } else {
#pragma unroll 1
                for (int c = col0; c < col0 + cols; c += 16) {
                    float o[16];
#pragma unroll
                    for (int y = 0; y < 16; ++y) o[y] = 0.0f;
                    uint32_t x[16];
                    if (have) {
                        tmem_ld_x16(t_o + first * D + c, x);
                        tmem_ld_wait();
                        if (c0 != 0.0f) {
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[y] = __uint_as_float(x[y]) * c0;
                        }
                    }
                    if (joined) {
                        tmem_ld_x16(t_o + D + c, x);
                        tmem_ld_wait();
                        if (c1 != 0.0f) {
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[y] = fmaf(__uint_as_float(x[y]), c1, o[y]);
                        }
                    }
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        *reinterpret_cast<float4*>(tile + lane * 64 + ((y ^ wsw) * 16)) = make_float4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
                    __syncwarp();
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const float4 q = *reinterpret_cast<const float4*>(tile + (y * 8 + lane / 4) * 64 + ((e ^ rsw) * 16));
                        if (to[y] >= 0) *reinterpret_cast<float4*>(a.part + to[y] + c + e * 4) = q;
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(o_empty);
                mbar_arrive(&u_empty[b]);
            }
            if (++b == 2) { b = 0; u_ph ^= 1u; }
        }
    }

done:
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && (warp == NSW + 1 || warp == NSW + 3) && lane == 0) tc_commit(drain_bar);
    if (warp == NSW + 1) {
        if (*abort_flag && lane == 0) {
            // gave up somewhere: let outstanding tensor-core work retire before TMEM goes away
            int dummy = 0;
            volatile int* never = &dummy;
            wait_bounded(drain_bar, 0, never, 73);
        }
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ---------------------------------------------------------------------------------------------- launch
// plan -> tcgen05 kernel (if any segment can be wide) -> few-row kernel -> join, one behind the other on the stream
template <int D, int HW, bool SELF>
static cudaError_t launch_attn_few(const AttnArgs& a, bool early, cudaStream_t st) {
    static PerDevice pd;
    constexpr int smem = FewCfg<D, HW, SELF>::SMEM;
    cudaError_t e = opt_in_shared_memory(pd, attn_few_kernel<D, HW, SELF>, smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(attn_few_kernel<D, HW, SELF>, dim3(a.few_ctas), dim3(AT_FEW_THREADS), smem, st, a, early);
}
// The kernel's register split only works out if it was compiled to be launched with AW_REGS_LAUNCH registers a thread.
template <int D>
static cudaError_t prepare_attn_wide() {
    static PerDevice pd;
    const int slot = per_device_slot();
    if (slot >= 0 && pd.done[slot]) return cudaSuccess;
    cudaFuncAttributes fa;
    cudaError_t e = cudaFuncGetAttributes(&fa, attn_wide_kernel<D>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs != AW_REGS_LAUNCH) return cudaErrorInvalidKernelImage;
    return opt_in_shared_memory(pd, attn_wide_kernel<D>, WideCfg<D>::SMEM);
}
template <int D>
static cudaError_t launch_attn_d(const AttnWideArgs& w, bool wide, cudaStream_t st) {
    const AttnArgs& a = w.a;
    cudaError_t e = wide ? prepare_attn_wide<D>() : cudaSuccess;
    if (e != cudaSuccess) return e;
    if (!wide && a.P == 0 && a.R <= FEW_SELF && a.few_hw == 4) {
        if ((e = launch_attn_few<D, 4, true>(a, false, st)) != cudaSuccess) return e;
    } else {
        const int threads = std::min(1024, std::max(128, (a.P + a.R + 31) / 32 * 32));
        if ((e = launch_pdl(attn_plan_kernel, dim3(1), dim3(threads), 0, st, a)) != cudaSuccess) return e;
        if (wide && (e = launch_pdl(attn_wide_kernel<D>, dim3(a.wide_ctas), dim3(AW_THREADS), WideCfg<D>::SMEM, st, w)) != cudaSuccess) return e;
        e = a.few_hw == 4 ? launch_attn_few<D, 4, false>(a, wide, st)
            : a.few_hw == 2 ? launch_attn_few<D, 2, false>(a, wide, st) : launch_attn_few<D, 1, false>(a, wide, st);
        if (e != cudaSuccess) return e;
    }
    JoinGrid g;
    g.wide_split = (int64_t)a.T * a.G >= 2048 ? 8 : 1;      // with few rows nearly all of them have two sources
    g.few_split = wide ? 1 : a.few_hw;
    g.wide_blocks = wide ? a.wide_ctas * g.wide_split : 0;
    g.row_blocks = a.P ? (int)std::min<int64_t>(3 * AT_MAX_SMS, ((int64_t)a.T * a.Hq + AT_JOIN_WARPS - 1) / AT_JOIN_WARPS) : 0;
    return launch_pdl((int64_t)a.T * a.Hq <= AT_JOIN_FEW_ROWS ? attn_join_kernel<D, 16> : attn_join_kernel<D, 8>,
                      dim3(g.row_blocks + g.wide_blocks + a.few_ctas * g.few_split), dim3(AT_JOIN_THREADS), 0, st, a, g);
}

cudaError_t launch_attn(const AttnWideArgs& w, int D, bool wide, cudaStream_t st) {
    return D == 128 ? launch_attn_d<128>(w, wide, st) : launch_attn_d<64>(w, wide, st);
}

}  // namespace osc
