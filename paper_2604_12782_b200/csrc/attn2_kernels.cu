// Attention for segments with many rows per key/value head (a prefix under many requests, a piece of a prompt):
// tcgen05 kernel on the tile line of attn_kernels.cu.
//
// A unit is two tiles of up to 128 rows (tokens x query heads of one key/value head).  S = Q K^T and O += P V
// both run on the fifth-generation tensor cores: Q, K and V tiles come by TMA into shared memory, S and O live in TMEM, P goes
// back into the columns of its S and is read from there as the A operand.  With D = 128 a 128 x 128 tile costs the tensor
// pipe 2 x 512 cycles and the exponential units (16 a cycle) 1024, so two streams run in counterphase, each with its
// own S, O and warpgroup (one row per thread): while one stream's softmax runs, the other's products do.
//   both row tiles filled: stream s is row tile s; they share every K and V tile.
//   one row tile:          both streams take the same rows and every other key tile; the results are joined
//                          at the end of the unit (a thread of warpgroup 0 can read both O rows: they lie in its lanes).
//
//   warps 0-3, 4-7 : softmax of stream 0, 1, and their epilogue
//   warp 8         : TMA (a key tile is loaded page by page; a page that is not there reads as zeros)
//   warp 9         : MMA issue, TMEM owner
//   warp 10        : the units of the CTA's share, for everyone else
//   warp 11        : idle; the third warpgroup gives registers to the softmax
//
// P V with the weights of the running maximum as it stands: O is rescaled in TMEM only when the maximum has moved by
// more than 2^8 (see AT_SLACK), by the softmax threads themselves.  That needs no wait of its own: the S tile that moved
// the maximum was issued behind the previous P V, so S complete means O complete.
#include <algorithm>

#include "common.cuh"

namespace osc {

struct AttnWideArgs {
    CUtensorMap tm_q;     // [T][Hq][D], box 64 channels x G heads x whole tokens of a tile
    CUtensorMap tm_k;     // [n_pages][Hk][page][D], box 64 channels x min(page, 128) tokens of one head
    CUtensorMap tm_v;
    AttnArgs a;
};

constexpr int AW_THREADS = 384;
// Registers: launched with 168 a thread (12 warps); the softmax warpgroups hold a row of 128 scores each thread and take
// 208, the third warpgroup (TMA, MMA, two idle warps) gives down to 80: 256 x 208 + 128 x 80 <= 384 x 168.
constexpr int AW_REGS_SOFTMAX = 208, AW_REGS_OTHER = 80;
template <int R>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack2(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D>
struct WideCfg {
    static constexpr int HALVES = D / 64;                        // 128-byte swizzle rows hold 64 channels
    static constexpr int HALF_BYTES = 128 * 128;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;       // 128 rows (or keys) x D
    static constexpr int STAGES = D == 128 ? 5 : 8;
    static constexpr int BAR_BYTES = 384;
    static constexpr int SMEM = (2 + STAGES) * TILE_BYTES + BAR_BYTES + 128 * 8 + 2 * 64 + 1024;
    static constexpr int TM_S = 0;         // TMEM columns: S0, S1, O0, O1
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
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                 "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
                 "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
                 "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
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

// What the roles need to know of a unit, or of the part of it that the CTA's share has: key tiles [ka, ka + n).  Warp 10
// walks over the line and keeps two of these ahead in shared memory.
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

__device__ __forceinline__ int unit_tile(const WideUnit& w, int s, int i) { return w.pair ? w.ka + i : w.ka + 2 * i + s; }
__device__ __forceinline__ int unit_load(const WideUnit& w, int s, int i) { return w.pair ? i : 2 * i + s; }   // which of the unit's K (or V) loads
// keys of key tile kt before any mask
__device__ __forceinline__ int unit_left(const WideUnit& w, int kt) {
    return kt < w.nf ? w.plen - kt * AT_WIDE_KEYS : w.klen - (kt - w.nf) * AT_WIDE_KEYS;
}

template <int D>
__global__ void __launch_bounds__(AW_THREADS, 1) attn_wide_kernel(const __grid_constant__ AttnWideArgs args) {
    using C = WideCfg<D>;
    constexpr int STAGES = C::STAGES;
    const AttnArgs& a = args.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring = smem + 2 * C::TILE_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + STAGES * C::TILE_BYTES);
    uint64_t* full = bars;
    uint64_t* empty = bars + STAGES;
    uint64_t* q_full = bars + 2 * STAGES;
    uint64_t* q_empty = q_full + 1;
    uint64_t* s_full = q_full + 2;
    uint64_t* p_full = q_full + 4;
    uint64_t* o_full = q_full + 6;
    uint64_t* o_empty = q_full + 8;
    uint64_t* j_full = q_full + 10;
    uint64_t* j_empty = q_full + 11;
    uint64_t* u_full = q_full + 12;      // [2]
    uint64_t* u_empty = q_full + 14;     // [2]
    uint64_t* drain_bar = q_full + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(q_full + 17);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float2* s_ml = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(bars) + C::BAR_BYTES);   // [128]: stream 1's (m, l)
    WideUnit* units = reinterpret_cast<WideUnit*>(s_ml + 128);                                   // [2]

    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&o_full[i], 1);
            mbar_init(&o_empty[i], 4);
            mbar_init(&u_full[i], 1);
            mbar_init(&u_empty[i], 10);
        }
        mbar_init(j_full, 4);
        mbar_init(j_empty, 4);
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&args.tm_q);
        prefetch_tmap(&args.tm_k);
        prefetch_tmap(&args.tm_v);
    }
    if (warp == 9) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
    grid_dependency_wait();
    grid_launch_dependents();   // not before: the few-row kernel counts on the plan being there when it begins
    const int tpt = AT_WIDE_TILE / a.G;

    if (warp >= 8) {
        regs_dec<AW_REGS_OTHER>();
        if (warp == 10) {
            // ------------------------------------------------------------------------------------- units
            const int S = a.P + a.R;
            const int64_t N = a.plan.wide_start[S], q = a.plan.share[1];
            const int64_t x0 = min(q * blockIdx.x, N), x1 = min(x0 + q, N);
            Cursor<WideUnits> cur;
            const LineSource<false> src = {a.plan.seg, a.plan.wide_start};
            if (x0 < x1) cur.seek(a, src, S, x0);
            else if (lane == 0) a.plan.cut[1][blockIdx.x].tiles = 0;
            int b = 0;
            uint32_t ph = 0;
            for (int64_t x = x0;;) {
                WideUnit w = {};
                if (x < x1) {
                    w.ka = cur.kt;
                    w.n = (int)min((int64_t)(cur.nt - cur.kt), x1 - x);
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
                    w.causal = cur.g.causal ? cur.g.n : 0;
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
                if (x < x1) cur.next_unit(a, src, SEG_WIDE);
            }
        } else if (warp == 8) {
            // --------------------------------------------------------------------------------------- TMA
            const int bt = min(1 << a.page_shift, AT_WIDE_KEYS);     // tokens of a box
            const int boxes = AT_WIDE_KEYS / bt * C::HALVES;         // of a K or V tile: at most 16, one lane each
            const int mine = lane / C::HALVES, half = lane % C::HALVES;
            const uint32_t ring0 = smem_u32(ring);
            uint32_t n_load = 0;            // loads so far: stage n % STAGES, phase n / STAGES
            int st = 0, b = 0;
            uint32_t ph = 0, q_ph = 0, u_ph = 0;
            while (true) {
                if (!wait_bounded(&u_full[b], u_ph, abort_flag, 60)) goto stop_loads;
                const WideUnit& w = units[b];
                const int ka = w.ka, kb = ka + w.n, nf = w.nf, h = w.h;
                if (kb == ka) break;
                if (!wait_bounded(q_empty, q_ph ^ 1u, abort_flag, 61)) goto stop_loads;
                q_ph ^= 1u;
                if (elect_one()) {
                    const int tiles = w.pair ? 2 : 1;
                    mbar_arrive_expect_tx(q_full, (uint32_t)(tiles * C::HALVES * tpt * a.G * 128));
                    for (int t = 0; t < tiles; ++t)
                        for (int hf = 0; hf < C::HALVES; ++hf)
                            tma_load_3d(smem_u32(smem + t * C::TILE_BYTES + hf * C::HALF_BYTES), &args.tm_q, q_full, hf * 64, h * a.G, w.row0 + t * tpt);
                }
                __syncwarp();
                const int32_t* own_pages = seg_pages(a, w.seg);
                const int32_t* front_pages = nf ? seg_pages(a, w.front) : own_pages;
                for (int kt = ka; kt < kb; ++kt) {
                    int page = a.n_pages, place = 0;      // a box past the last page is filled with zeros
                    if (lane < boxes) {
                        const int key = (kt < nf ? kt : kt - nf) * AT_WIDE_KEYS + mine * bt;
                        if (mine * bt < unit_left(w, kt)) {          // a length is within the list's columns
                            const int p = (kt < nf ? front_pages : own_pages)[key >> a.page_shift];
                            if (p >= 0 && p < a.n_pages) page = p;
                            place = key & ((1 << a.page_shift) - 1);
                        }
                    }
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        if (!wait_bounded(&empty[st], ph ^ 1u, abort_flag, 62)) goto stop_loads;
                        if (lane == 0) mbar_arrive_expect_tx(&full[st], C::TILE_BYTES);
                        __syncwarp();
                        if (lane < boxes)
                            tma_load_4d(ring0 + st * C::TILE_BYTES + half * C::HALF_BYTES + mine * bt * 128, kv ? &args.tm_v : &args.tm_k, &full[st],
                                        half * 64, place, h, page);
                        ++n_load;
                        if (++st == STAGES) { st = 0; ph ^= 1u; }
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
                for (uint32_t i = n_load > STAGES ? n_load - STAGES : 0; i < n_load; ++i)
                    wait_bounded(&full[i % STAGES], (i / STAGES) & 1u, never, 63);
                wait_bounded(q_full, q_ph ^ 1u, never, 64);
            }
        } else if (warp == 9) {
            // --------------------------------------------------------------------------------------- MMA
            const uint32_t ring0 = smem_u32(ring), q0 = smem_u32(smem);
            const uint64_t k_hi = smem_desc_sw128(0), v_hi = smem_desc_sw128_mn(0, C::HALVES > 1 ? C::HALF_BYTES : 1024);
            constexpr uint32_t IDESC_S = idesc_bf16(128, 128), IDESC_O = idesc_bf16(128, D) | IDESC_B_MN;
            uint32_t base = 0;                 // loads of the units before
            uint32_t q_ph = 0, p_ph[2] = {0, 0}, oe_ph[2] = {1, 1}, u_ph = 0;
            int b = 0;
            while (true) {
                if (!wait_bounded(&u_full[b], u_ph, abort_flag, 77)) goto done;
                const WideUnit& w = units[b];
                const int n = w.n, pair = w.pair, cnt[2] = {w.cnt[0], w.cnt[1]};
                if (n == 0) break;
                if (!wait_bounded(q_full, q_ph, abort_flag, 65)) goto done;
                q_ph ^= 1u;
                // S_s(i): product of the stream's rows with its i-th key tile
                auto issue_s = [&](int s, int i) -> bool {
                    const uint32_t ld = base + 2 * unit_load(w, s, i), stg = ld % STAGES;
                    if (!wait_bounded(&full[stg], (ld / STAGES) & 1u, abort_flag, 66)) return false;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t qa = q0 + (pair && s ? C::TILE_BYTES : 0), kb = ring0 + stg * C::TILE_BYTES;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = (k / 4) * C::HALF_BYTES + (k % 4) * 32;
                            mma_f16(tmem + C::TM_S + s * 128, k_hi | (uint64_t)((qa + off) >> 4), k_hi | (uint64_t)((kb + off) >> 4), IDESC_S, k ? 1u : 0u);
                        }
                        tc_commit(&s_full[s]);
                        if (!pair || s == 1) tc_commit(&empty[stg]);
                    }
                    __syncwarp();
                    return true;
                };
                for (int s = 0; s < 2; ++s)
                    if (cnt[s] > 0 && !issue_s(s, 0)) goto done;
                const int most = max(cnt[0], cnt[1]);
                for (int i = 0; i < most; ++i) {
                    for (int s = 0; s < 2; ++s) {
                        if (i >= cnt[s]) continue;
                        if (i == 0) {      // the epilogue of the unit before has read O
                            if (!wait_bounded(&o_empty[s], oe_ph[s], abort_flag, 67)) goto done;
                            oe_ph[s] ^= 1u;
                        }
                        const uint32_t ld = base + 2 * unit_load(w, s, i) + 1, stg = ld % STAGES;
                        if (!wait_bounded(&full[stg], (ld / STAGES) & 1u, abort_flag, 68)) goto done;
                        const int left = unit_left(w, unit_tile(w, s, i));
                        if (left < AT_WIDE_KEYS && (s == 0 || !pair || i >= cnt[0])) {
                            // Behind the last key the page holds whatever was there before: a NaN or Inf would survive its weight of 0.
                            uint8_t* v = ring + stg * C::TILE_BYTES;
                            for (int c = left * 8 + lane; c < AT_WIDE_KEYS * 8; c += 32)
#pragma unroll
                                for (int hf = 0; hf < C::HALVES; ++hf)
                                    *reinterpret_cast<uint4*>(v + hf * C::HALF_BYTES + c * 16) = make_uint4(0u, 0u, 0u, 0u);
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                        if (!wait_bounded(&p_full[s], p_ph[s], abort_flag, 69)) goto done;
                        p_ph[s] ^= 1u;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t vb = ring0 + stg * C::TILE_BYTES;
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                mma_f16_ts(tmem + C::TM_O + s * D, tmem + C::TM_S + s * 128 + k * 8, v_hi | (uint64_t)((vb + k * 2048) >> 4), IDESC_O,
                                           (i | k) ? 1u : 0u);
                            if (!pair || s == 1) tc_commit(&empty[stg]);
                            if (i == cnt[s] - 1) tc_commit(&o_full[s]);
                        }
                        __syncwarp();
                        if (i + 1 < cnt[s] && !issue_s(s, i + 1)) goto done;
                    }
                }
                if (elect_one()) tc_commit(q_empty);
                __syncwarp();
                base += 2 * (uint32_t)n;
                if (lane == 0) mbar_arrive(&u_empty[b]);
                if (++b == 2) { b = 0; u_ph ^= 1u; }
            }
        }
    } else {
        // ------------------------------------------------------------------------------------------ softmax
        regs_inc<AW_REGS_SOFTMAX>();
        const int s = warp >> 2;
        const int r = threadIdx.x & 127;                                 // row of the tile = TMEM lane
        const int my_tok = r / a.G, my_head = r % a.G;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + C::TM_S + s * 128, t_o = tmem + lanes + C::TM_O;
        uint32_t s_ph = 0, o_ph[2] = {0, 0}, j_ph = 0, u_ph = 0;
        int b = 0;
        while (true) {
            if (!wait_bounded(&u_full[b], u_ph, abort_flag, 78)) goto done;
            const WideUnit& w = units[b];
            if (w.n == 0) break;
            float m = -INFINITY, l = 0.0f;
            {
                const int tok = (w.pair ? s * tpt : 0) + my_tok;         // token inside the unit
                const bool valid = my_tok < tpt && tok < w.tokens;
                const int nf = w.nf, step = w.pair ? 1 : 2;
                // keys that the row sees from the first key of the own tile 0 on; a row that is not there sees all
                const int sees = valid && w.causal ? max(w.klen - w.causal + w.tok0 + tok + 1, 0) : w.klen;
                int kt = w.pair ? w.ka : w.ka + s;
                for (int i = 0, cnt = w.cnt[s]; i < cnt; ++i, kt += step) {
                    if (!wait_bounded(&s_full[s], s_ph, abort_flag, 70)) goto done;
                    s_ph ^= 1u;
                    tc_fence_after();
                    uint32_t v[4][32];
#pragma unroll
                    for (int j = 0; j < 4; ++j) tmem_ld_32x32(t_s + j * 32, v[j]);
                    tmem_ld_wait();
                    const int left = kt < nf ? w.plen - kt * AT_WIDE_KEYS : sees - (kt - nf) * AT_WIDE_KEYS;   // keys of the tile that the row sees
                    if (!__all_sync(0xFFFFFFFFu, left >= AT_WIDE_KEYS)) {
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
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
                    float f = 1.0f;
                    const bool move = top > m + AT_SLACK;
                    if (move) {
                        f = exp2_approx(m - top);
                        m = top;
                        l *= f;
                    }
                    const float ref = m == -INFINITY ? 0.0f : -m;
                    const uint64_t scale2 = pack2(a.scale_log2, a.scale_log2), ref2 = pack2(ref, ref);
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float p0, p1;
                            unpack2(fma2(pack2(__uint_as_float(v[j][e]), __uint_as_float(v[j][e + 1])), scale2, ref2), p0, p1);
                            p0 = exp2_approx(p0);
                            p1 = exp2_approx(p1);
                            sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pack2(p0, p1));
                            pk[e / 2] = bf162_bits(__floats2bfloat162_rn(p0, p1));
                        }
                        tmem_st_32x16(t_s + j * 16, pk);
                    }
                    float s0, s1;
                    unpack2(add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    if (__any_sync(0xFFFFFFFFu, move) && i > 0) {
#pragma unroll
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            tmem_ld_32x32(t_o + s * D + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st_32x32(t_o + s * D + c, o);
                        }
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[s]);
                }
            }
            // ---- the unit's rows: into O, or as (m, l, O) into the workspace
            const bool pair = w.pair, have0 = w.cnt[0] > 0, have1 = w.cnt[1] > 0, have = s ? have1 : have0;
            float m1 = -INFINITY, l1 = 0.0f;
            if (!pair) {
                if (s == 1) {
                    if (!wait_bounded(j_empty, j_ph ^ 1u, abort_flag, 74)) goto done;
                    s_ml[r] = make_float2(m, l);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(j_full);
                } else {
                    if (!wait_bounded(j_full, j_ph, abort_flag, 75)) goto done;
                    m1 = s_ml[r].x;
                    l1 = s_ml[r].y;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(j_empty);
                }
                j_ph ^= 1u;
            }
            if (pair || s == 0) {
                const bool two = !pair && have1;
                if (have && !wait_bounded(&o_full[s], o_ph[s], abort_flag, 71)) goto done;
                if (two && !wait_bounded(&o_full[1], o_ph[1], abort_flag, 72)) goto done;
                tc_fence_after();
                const int tok = (pair ? s * tpt : 0) + my_tok, hq = w.h * a.G + my_head, out = w.out;
                const bool valid = my_tok < tpt && tok < w.tokens;
                const float mn = fmaxf(m, m1);
                const float f0 = mn == -INFINITY ? 0.0f : exp2_approx(m - mn), f1 = mn == -INFINITY ? 0.0f : exp2_approx(m1 - mn);
                const float lt = l * f0 + l1 * f1;
                const bool direct = !(out & (OUT_SPLIT | OUT_TWO));
                const float inv = !direct ? 1.0f : lt > 0.0f || lt != lt ? 1.0f / lt : 0.0f;
                const float c0 = f0 * inv, c1 = f1 * inv;
                const int64_t token = w.row0 + tok, row = token * a.Hq + hq;
                const int64_t at = out & OUT_SPLIT ? ((int64_t)blockIdx.x * 2 + (out & OUT_LATER ? 1 : 0)) * (2 * AT_WIDE_TILE) + (pair ? s * AT_WIDE_TILE : 0) + r : row;
                float* part = (out & OUT_SPLIT ? a.wide_part : a.dense[out & OUT_OWN ? 1 : 0]) + at * D;
                uint16_t* op = a.o + token * a.ldo + (int64_t)hq * D;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    if (have) {
                        tmem_ld_32x32(t_o + s * D + c, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = have && c0 != 0.0f ? __float_as_uint(__uint_as_float(o[e]) * c0) : 0u;
                    if (two) {
                        uint32_t o1[32];
                        tmem_ld_32x32(t_o + D + c, o1);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(fmaf(__uint_as_float(o1[e]), c1, __uint_as_float(o[e])));
                    }
                    if (valid) {
                        if (direct) {
#pragma unroll
                            for (int e = 0; e < 32; e += 8) {
                                uint32_t h[4];
#pragma unroll
                                for (int y = 0; y < 4; ++y)
                                    h[y] = bf162_bits(__floats2bfloat162_rn(__uint_as_float(o[e + 2 * y]), __uint_as_float(o[e + 2 * y + 1])));
                                *reinterpret_cast<uint4*>(op + c + e) = make_uint4(h[0], h[1], h[2], h[3]);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                *reinterpret_cast<uint4*>(part + c + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                        }
                    }
                }
                if (valid) {
                    if (!direct) (out & OUT_SPLIT ? a.wide_ml : a.dense_ml[out & OUT_OWN ? 1 : 0])[at] = make_float2(mn, lt);
                    else if (a.lse) a.lse[row] = lt == 0.0f ? -INFINITY : (mn + log2f(lt)) * 0.69314718055994531f;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (have) mbar_arrive(&o_empty[s]);
                    if (two) mbar_arrive(&o_empty[1]);
                }
            }
            o_ph[0] ^= have0;
            o_ph[1] ^= have1;
            __syncwarp();
            if (lane == 0) mbar_arrive(&u_empty[b]);
            if (++b == 2) { b = 0; u_ph ^= 1u; }
        }
    }

done:
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        if (*abort_flag && lane == 0) {
            // gave up somewhere: let outstanding tensor-core work retire before TMEM goes away
            tc_commit(drain_bar);
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
template <int D>
static cudaError_t launch_attn_d(const AttnWideArgs& w, bool wide, cudaStream_t st) {
    static PerDevice pd_wide;
    const AttnArgs& a = w.a;
    cudaError_t e = wide ? opt_in_shared_memory(pd_wide, attn_wide_kernel<D>, WideCfg<D>::SMEM) : cudaSuccess;
    if (e != cudaSuccess) return e;
    if (!wide && a.P == 0 && a.R <= FEW_SELF && a.few_hw == 4) {
        if ((e = launch_attn_few<D, 4, true>(a, false, st)) != cudaSuccess) return e;
    } else {
        const int threads = std::min(1024, std::max(128, (a.P + a.R + 127) / 128 * 128));
        if ((e = launch_pdl(attn_plan_kernel, dim3(1), dim3(threads), 0, st, a)) != cudaSuccess) return e;
        if (wide && (e = launch_pdl(attn_wide_kernel<D>, dim3(a.wide_ctas), dim3(AW_THREADS), WideCfg<D>::SMEM, st, w)) != cudaSuccess) return e;
        e = a.few_hw == 4 ? launch_attn_few<D, 4, false>(a, wide, st)
            : a.few_hw == 2 ? launch_attn_few<D, 2, false>(a, wide, st) : launch_attn_few<D, 1, false>(a, wide, st);
        if (e != cudaSuccess) return e;
    }
    const int wide_split = 8, few_split = a.few_hw;
    const int wide_blocks = wide ? a.wide_ctas * wide_split : 0, few_blocks = a.few_ctas * few_split;
    const int tokens = (int)std::min<int64_t>(32, std::max<int64_t>(1, (int64_t)a.T * a.Hk / (4 * AT_MAX_SMS)));
    const int64_t token_blocks = a.P ? ((int64_t)a.T + tokens - 1) / tokens * a.Hk : 0;
    if (wide_blocks + few_blocks + token_blocks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    return launch_pdl(attn_join_kernel<D>, dim3((unsigned)(wide_blocks + few_blocks + token_blocks)), dim3(AT_JOIN_THREADS), 0, st, a, wide_blocks,
                      wide_split, few_blocks, few_split, tokens);
}

cudaError_t launch_attn(const AttnWideArgs& w, int D, bool wide, cudaStream_t st) {
    return D == 128 ? launch_attn_d<128>(w, wide, st) : launch_attn_d<64>(w, wide, st);
}

}  // namespace osc
