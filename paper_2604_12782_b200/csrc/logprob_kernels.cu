// Log probabilities of given tokens, log-sum-exp, entropy and the best alternatives of every row of logits, in one pass.
//
//   d_j = x_j - max x,  l = sum_j exp(scale d_j),  S = sum_j d_j exp(scale d_j)
//   lse = scale max x + ln l,   log p_j = scale d_j - ln l,   entropy = ln l - scale S / l
//
// For a scale so small that logits near the end of fp32's range still count (below 10^-20: no difference that has a weight passes 10^22 otherwise, nor does a sum
// of 2^30 of them end the range) differences and S are held in units of 2^40 (SMALL: kernels of their own, whose loop takes values one by one).
//
// ln l and -S are never negative, so nothing cancels where a row is sure of one token.  But l is then just above 1, and every addition to a sum that holds the
// 1 rounds what is above it to 2^-24.  Where l comes out below 1 + 2^-7, the warp whose thread has the maximum goes over that thread's values (one part of
// as many as the row has threads) once more without it, and what is above 1 is summed by itself; ln l is then log1p of that.  A thread keeps its own (max, l, S) and joins a
// chunk of 16-byte vectors at a time: the chunk's maximum first, one correction of (l, S) if it is a new one, then the chunk's terms
// (l' = l f, S' = f (S + l (m - m')), f = exp(scale (m - m'))).  A row is one block's, or with few rows a cluster's, whose blocks take
// consecutive parts and are joined through distributed shared memory, so there is one launch and no workspace.  Every thread copies its own
// vectors into a ring in shared memory (cp.async), two chunks ahead; nobody else reads them, so the ring needs no barrier.
//
// Alternatives: the order is value, then lower index, as one key: the value's bits made monotone (NaN below -inf) and the index.  The loop over the
// chunks keeps nothing but the largest key of every eight threads' part of a chunk (256 values), in short rows of every thread's (32).  Behind it, the k-th largest of those bounds the k-th best value
// of the row from below, so the best are in the parts that reach it, about k of them: these are read again (from L2 mostly) and their values at or
// above the bound, a few more than k, are ranked.  No barrier runs in the loop, and the maxima take 15 instructions of a warp and chunk.  (Candidates picked out of every chunk as
// it passed, with a bound that rose, took 60 more: 240 us for 3001 rows of 152064 bf16 logits.)  Where too many values reach the bound (equal logits), or too
// few parts have any (short rows, masks), the chunks are read again in order, each with a bound of its own; chunks whose largest value is not above the k-th
// so far are passed over, and where ties alone fill the list a chunk's best are taken one by one, k rounds of a maximum over the block.
//
// Bound: without alternatives HBM (3001 rows of 152064 bf16 logits 150 us, 0.93 of the copy rate), with 20 of them the issue of instructions (189 us, 0.73: 3.1 of 4 slots a
// cycle, of which the exponentials' conversions, products and sums are most); 1500 such rows of fp32, half as many values to a byte, 149 us, 0.93.  Few rows:
// latency, 26 rows of 128000 in fp32 12.4 us, 2.0 at the copy rate.  Two rules on sizes.  Rows of up to 16 KB are on blocks of two warps: a block of
// eight has less than a chunk of them, and the steps behind the loop, which cost a block the same whatever the row, bound them (with 20 alternatives 20000 rows of
// 4096 in bf16 234 us with eight warps, 131 with two, of 8192, the longest that count as short, 250 and 161).  Rows that do not fill the machine are split over
// clusters of up to eight (one row of 151936 in fp32 26.8 us without, 12.6 with; 220 of them in bf16, the most that still are, 26.9 and 24.8).
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"

namespace osc {

constexpr int LP_VECS = 4;               // 16-byte vectors of a chunk, per thread
static_assert(LP_VECS * 8 <= 32, "a lane for every value of a thread");
constexpr int LP_STAGES = 3;             // chunks in the ring
constexpr int LP_SHORT_BYTES = 16384;    // rows up to here
constexpr int LP_PARTS = 1024;           // parts of a block's row
constexpr float LP_SURE = 1.0f + 1.0f / 128;
constexpr int LP_MAX_TOP = 32;
constexpr int LP_LIST = 512;            // candidates that wait to be ranked
constexpr int LP_MAX_CLUSTER = 8;

struct LogprobArgs {
    const void* x;
    int64_t ld;
    const int32_t* ids;
    int64_t ld_ids;
    float* logprob;          // [T][n_ids]
    float* lse;              // may be null
    float* entropy;          // may be null
    int32_t* top_ids;        // [T][k]
    float* top_logprob;
    int T, V, n_ids, k;
    float scale;
};

// A value's place in the order: 0 is no value at all, 1 a NaN, then rising from -inf; -0 and 0 are equal.
__device__ __forceinline__ uint32_t lp_key(float x) {
    if (x != x) return 1u;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t LP_KEY_LOW = 0x007FFFFFu;      // -inf
__device__ __forceinline__ float lp_value(uint32_t key) {
    if (key <= 1u) return __uint_as_float(0x7FC00000u);
    return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
// key in the high half, complement of the index in the low one: larger is better, and no two are equal
__device__ __forceinline__ unsigned long long lp_rank(uint32_t key, int idx) { return (unsigned long long)key << 32 | (uint32_t)~idx; }

__device__ __forceinline__ float lp_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool F32>
struct LpVec {
    static constexpr int E = F32 ? 4 : 8;            // elements of a vector
    using Elem = typename std::conditional<F32, float, uint16_t>::type;
    __device__ static float value(Elem x) { return F32 ? (float)x : __uint_as_float((uint32_t)x << 16); }
    // element e of a vector; e is known when compiling
    __device__ static float get(const uint4& v, int e) {
        const uint32_t w = F32 ? (e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w) : (e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w);
        return __uint_as_float(F32 ? w : e & 1 ? w & 0xFFFF0000u : w << 16);
    }
};

template <bool F32, bool TOP, int NT, bool SMALL>
__global__ void __launch_bounds__(NT, 1024 / NT) token_logprobs_kernel(const LogprobArgs a, int cluster) {
    using Vec = LpVec<F32>;
    using Elem = typename Vec::Elem;
    constexpr int E = Vec::E, U = LP_VECS, CHUNK = NT * U, WARPS = NT / 32;
    extern __shared__ __align__(16) uint8_t lp_ring[];       // [LP_STAGES][CHUNK] vectors
    __shared__ unsigned long long s_kept[2][TOP ? LP_MAX_TOP : 1];       // the k best, in order (0: none); the one of two that `which` says
    __shared__ unsigned long long s_warp[WARPS];
    __shared__ float s_red[3][WARPS];
    __shared__ unsigned long long s_in[TOP ? LP_MAX_CLUSTER * LP_MAX_TOP : 1];     // the k best of the cluster's other blocks, in the one of rank 0
    __shared__ float s_part[LP_MAX_CLUSTER][4];      // (max, l, S, l - 1) of the cluster's blocks, likewise
    __shared__ uint32_t s_most[TOP ? LP_PARTS : 1];                       // largest key above -inf of every part
    // behind the loop the ring holds
    unsigned long long* s_list = reinterpret_cast<unsigned long long*>(lp_ring);       // candidates
    uint16_t* s_part_of = reinterpret_cast<uint16_t*>(s_list + LP_LIST);               // [LP_PARTS] the parts that reach the bound
    __shared__ int s_parts;
    __shared__ int s_n, s_over;                      // candidates; whether some found no place
    grid_launch_dependents();
    if (cluster > 1) cluster_meet();                 // every block is there before anyone writes to rank 0
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = cluster > 1 ? (int)cluster_ctarank() : 0;
    const int64_t row = blockIdx.x / cluster;
    constexpr float UNIT = SMALL ? 0x1p-40f : 1.0f;              // differences are held as x UNIT - max UNIT
    const float rate = SMALL ? a.scale * 0x1p40f : a.scale, scale2 = rate * 1.44269504088896341f;
    auto diff = [&](float x, float from) { return SMALL ? x * UNIT - from * UNIT : x - from; };
    const int k = TOP ? a.k : 0;
    if (TOP) {
        if (tid == 0) s_n = s_over = s_parts = 0;
        if (tid < 2 * LP_MAX_TOP) s_kept[tid / LP_MAX_TOP][tid % LP_MAX_TOP] = 0;
    }
    grid_dependency_wait();

    // Rows begin at any element: vectors are counted from the 16-byte boundary at or before the row, whose first `lead` elements are not the row's.
    // Vectors [full0, full1) are the row's as a whole, [v0, v1) of them this block's; the few elements in front and behind come last.
    const Elem* xr = static_cast<const Elem*>(a.x) + row * a.ld;
    const int lead = (int)((reinterpret_cast<uintptr_t>(xr) & 15u) / sizeof(Elem));
    const uint4* xv = reinterpret_cast<const uint4*>(xr - lead);
    const int full0 = lead ? 1 : 0, full1 = max((int)(((int64_t)lead + a.V) / E), full0);
    const int v0 = full0 + (int)((int64_t)(full1 - full0) * rank / cluster), v1 = full0 + (int)((int64_t)(full1 - full0) * (rank + 1) / cluster);

    uint4* mine = reinterpret_cast<uint4*>(lp_ring) + tid;       // the thread's vectors of a stage: mine[u * NT]
    const uint64_t policy = l2_policy_evict_first();             // read once
    auto load = [&](int base, int stage) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * NT + tid;
            if (i < v1) cp_async_16(smem_u32(mine + stage * CHUNK + u * NT), xv + i, true, policy);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < LP_STAGES - 1; ++i) load(v0 + i * CHUNK, i);

    float m = -INFINITY, l = 0.0f, S = 0.0f;
    uint32_t bound = 0;          // values with a key above it are candidates
    int which = 0;
    if (TOP) __syncthreads();

    // Joins the candidates with the k best; `bound` becomes the last one's key.  All threads have passed a barrier since the last candidate came.
    auto rank_list = [&](const unsigned long long* list, int n) {
        unsigned long long* to = s_kept[which ^ 1];
        const unsigned long long* from = s_kept[which];
        // four lanes to an entry, which share out the others
#pragma unroll 1
        for (int i0 = 0; i0 < n + k; i0 += NT / 4) {
            const int i = i0 + tid / 4;
            const unsigned long long x = i < k ? from[i] : i < n + k ? list[i - k] : 0;
            int better = 0;
#pragma unroll 2
            for (int j = tid & 3; j < k; j += 4) better += from[j] > x;
#pragma unroll 4
            for (int j = tid & 3; j < n; j += 4) better += list[j] > x;
            better += __shfl_xor_sync(0xFFFFFFFFu, better, 1);
            better += __shfl_xor_sync(0xFFFFFFFFu, better, 2);
            if (x != 0 && better < k) to[better] = x;
        }
        __syncthreads();
        which ^= 1;
        bound = (uint32_t)(s_kept[which][k - 1] >> 32);
        if (tid < k) s_kept[which ^ 1][tid] = 0;
        if (tid == 0) s_n = s_over = 0;
        __syncthreads();
    };
    auto add = [&](uint32_t key, int j) {
        const int n = atomicAdd(&s_n, 1);
        if (n < LP_LIST) s_list[n] = lp_rank(key, j);
        else s_over = 1;
    };
    // every value of the thread in a chunk, which lies at `at` (NT vectors apart): f(key, index)
    auto each = [&](const uint4* at, int base, auto f) {
#pragma unroll 1
        for (int u = 0; u < U && base + u * NT + tid < v1; ++u) {
            const uint4 x = at[u * NT];
            const int j = (base + u * NT + tid) * E - lead;
#pragma unroll
            for (int e = 0; e < E; ++e) f(lp_key(Vec::get(x, e)), j + e);
        }
    };
    // the largest 16-bit prefix of a key that k threads' largest ones reach; 0: fewer have any
    auto reached = [&](uint32_t best) -> uint32_t {
        uint32_t t = 0;
#pragma unroll 1
        for (int bit = 15; bit >= 0; --bit)
            if (__syncthreads_count(best >> 16 >= (t | 1u << bit)) >= k) t |= 1u << bit;
        return t << 16;
    };
    // the values of a chunk above the bound, joined with the k best
    auto again = [&](int base) {
        const uint4* at = xv + base + tid;
        uint32_t best = 0;
        each(at, base, [&](uint32_t key, int) { best = max(best, key); });
        const uint32_t t = reached(best);
        if (t) bound = max(bound, t - 1);
        each(at, base, [&](uint32_t key, int j) { if (key > bound) add(key, j); });
        __syncthreads();
        if (!s_over) return rank_list(s_list, s_n);
        __syncthreads();
        if (tid == 0) s_n = 0;
        __syncthreads();
        bound = (uint32_t)(s_kept[which][k - 1] >> 32);
        unsigned long long last = ~0ull;
#pragma unroll 1
        for (int i = 0; i < k; ++i) {
            unsigned long long next = 0;
            each(at, base, [&](uint32_t key, int j) {
                const unsigned long long c = lp_rank(key, j);
                if (c < last && c > next) next = c;
            });
#pragma unroll
            for (int o = 16; o; o >>= 1) next = max(next, __shfl_xor_sync(0xFFFFFFFFu, next, o));
            if (lane == 0) s_warp[warp] = next;
            __syncthreads();
            last = s_warp[0];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) last = max(last, s_warp[w]);
            __syncthreads();
            if ((uint32_t)(last >> 32) <= bound) break;      // 0, or no better than the k of the chunks before
            if (tid == 0) s_list[s_n++] = last;
        }
        __syncthreads();
        rank_list(s_list, s_n);
    };

    // ---- the elements in front of the row's first whole vector and behind its last one
    const int head = min(full0 * E - lead, a.V), tail = max(full1 * E - lead, head);          // [0, head), [tail, V)
    const int edge = rank == 0 && tid < head ? tid : rank == cluster - 1 && tid >= 32 && tid - 32 < a.V - tail ? tail + tid - 32 : -1;
    if (edge >= 0) {
        const float x = Vec::value(xr[edge]);
        if (x != -INFINITY) {
            m = x != x ? -INFINITY : x;
            l = lp_exp2((x - x) * scale2);           // 1, or NaN
        }
    }

    int stage = 0, chunk = 0;
    const int chunks = (v1 - v0 + CHUNK - 1) / CHUNK;
    int shift = 0;               // of chunks to the groups of them whose parts are one
    while (chunks >> shift >= LP_PARTS / (NT / 8)) ++shift;
    const bool fine = chunks * NT <= LP_PARTS;       // a part is a thread's
#pragma unroll 1
    for (int base = v0; base < v1; base += CHUNK, ++chunk) {
        // into the stage of the chunk before, whose vectors are done with
        load(base + (LP_STAGES - 1) * CHUNK, stage == 0 ? LP_STAGES - 1 : stage - 1);
        cp_async_wait<LP_STAGES - 1>();
        const uint4* at = mine + stage * CHUNK;
        stage = stage + 1 == LP_STAGES ? 0 : stage + 1;
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u].x = v[u].y = v[u].z = v[u].w = F32 ? 0xFF800000u : 0xFF80FF80u;      // past the end: -inf
            if (base + u * NT + tid < v1) v[u] = at[u * NT];
        }
        // ---- the chunk's maximum (a NaN leaves it alone)
        float top;
        if (F32) {
            top = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, fmaxf(fmaxf(Vec::get(v[u], 0), Vec::get(v[u], 1)), fmaxf(Vec::get(v[u], 2), Vec::get(v[u], 3))));
        } else {
            __nv_bfloat162 t = __halves2bfloat162(__ushort_as_bfloat16(0xFF80), __ushort_as_bfloat16(0xFF80));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
                const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(w);
                t = __hmax2(t, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
            }
            top = fmaxf(__low2float(t), __high2float(t));
        }
        // ---- (max, l, S)
        if (top > m) {
            if (m > -INFINITY) {
                const float d = diff(m, top), f = lp_exp2(d * scale2);
                S = f == 0.0f ? 0.0f : f * (S + l * d);      // d may be -inf
                l *= f;
            }
            m = top;
        }
        {
            // A thread without a value above -inf has nothing to add; but a NaN has to reach the sums.
            const float ref = m == -INFINITY ? 0.0f : -(m * UNIT);
            float sum = 0.0f;
            if (!SMALL) {
                const uint64_t ref2 = pack2(ref, ref), sc2 = pack2(scale2, scale2);
                uint64_t lc = 0, sc = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (base + u * NT + tid >= v1) break;
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const uint64_t d = add2(pack2(Vec::get(v[u], e), Vec::get(v[u], e + 1)), ref2);
                        float t0, t1;
                        unpack2(mul2(d, sc2), t0, t1);
                        const uint64_t p = pack2(lp_exp2(t0), lp_exp2(t1));
                        lc = add2(lc, p);
                        sc = fma2(p, d, sc);
                    }
                }
                float l0, l1, s0, s1;
                unpack2(lc, l0, l1);
                unpack2(sc, s0, s1);
                l += l0 + l1;
                sum = s0 + s1;
            }
            if (SMALL || sum != sum) {        // 0 * -inf: -inf among the logits (or a NaN, or +inf, which l shows)
                float more = 0.0f;
                sum = 0.0f;
#pragma unroll 1
                for (int u = 0; u < U && base + u * NT + tid < v1; ++u) {
                    const uint4 x = at[u * NT];
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float d = Vec::get(x, e) * UNIT + ref, p = lp_exp2(d * scale2);
                        more += p;
                        sum += p == 0.0f ? 0.0f : p * d;
                    }
                }
                if (SMALL) l += more;
            }
            S += sum;
        }
        if (TOP) {
            const uint32_t key = top > -INFINITY ? lp_key(top) : 0u;
            if (fine) {
                s_most[chunk * NT + tid] = key;
            } else {
                uint32_t most = key;
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
                if ((lane & 7) == 0) {
                    uint32_t* to = &s_most[(chunk >> shift) * (NT / 8) + tid / 8];
                    *to = chunk & ((1 << shift) - 1) ? max(*to, most) : most;
                }
            }
        }
    }
    cp_async_wait<0>();

    // ---- the k best of the block's part
    if (TOP) {
        const int parts = fine ? chunks * NT : (((chunks - 1) >> shift) + 1) * (NT / 8);
        __syncthreads();
        uint32_t best = 0;
        for (int i = tid; i < parts; i += NT) best = max(best, s_most[i]);
        const uint32_t t = reached(best);
        bool done = false;
        if (t) {
            for (int i = tid; i < parts; i += NT)
                if (s_most[i] >= t) s_part_of[atomicAdd(&s_parts, 1)] = (uint16_t)i;
            __syncthreads();
            const int n = s_parts;
            constexpr int FLIGHT = 4;        // parts whose values are on their way
#pragma unroll 1
            for (int i0 = warp; fine && i0 < n; i0 += FLIGHT * WARPS) {       // a lane for every value
                Elem x[FLIGHT];
                int j[FLIGHT];
#pragma unroll
                for (int f = 0; f < FLIGHT; ++f) {
                    const int i = i0 + f * WARPS, part = s_part_of[min(i, n - 1)], u = lane / E;
                    const int at = v0 + part / NT * CHUNK + u * NT + part % NT;
                    j[f] = i < n && u < U && at < v1 ? at * E + lane % E - lead : -1;
                    x[f] = j[f] >= 0 ? xr[j[f]] : Elem(0);
                }
#pragma unroll
                for (int f = 0; f < FLIGHT; ++f) {
                    const uint32_t key = lp_key(Vec::value(x[f]));
                    if (j[f] >= 0 && key >= t) add(key, j[f]);
                }
            }
            const float least = lp_value(t);         // (t is above the -inf of what is not there, and a NaN is not at or above anything)
            const int per = 8 * U << shift, total = fine ? 0 : n * per;          // vectors of a part, of all
            constexpr int VECS = 3;
#pragma unroll 1
            for (int i0 = tid; i0 < total; i0 += VECS * NT) {
                uint4 x[VECS];
                int at[VECS];
#pragma unroll
                for (int f = 0; f < VECS; ++f) {
                    const int i = i0 + f * NT, part = s_part_of[min(i, total - 1) / per], r = i % per;
                    const int c = (part / (NT / 8) << shift) + r / (8 * U);
                    at[f] = v0 + c * CHUNK + r / 8 % U * NT + part % (NT / 8) * 8 + r % 8;
                    x[f].x = x[f].y = x[f].z = x[f].w = F32 ? 0xFF800000u : 0xFF80FF80u;
                    if (i < total && at[f] < v1) x[f] = xv[at[f]];
                }
#pragma unroll
                for (int f = 0; f < VECS; ++f)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float y = Vec::get(x[f], e);
                        if (y >= least) add(lp_key(y), at[f] * E + e - lead);
                    }
            }
            if (edge >= 0) add(lp_key(Vec::value(xr[edge])), edge);
            __syncthreads();
            done = !s_over;
            if (done) rank_list(s_list, s_n);
        }
        if (!done) {
            __syncthreads();
            if (tid == 0) s_n = s_over = 0;
            __syncthreads();
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                uint32_t most = 0;
                if (fine) {
                    const uint32_t key = s_most[c * NT + tid];
                    most = __syncthreads_or(key > bound) ? 0xFFFFFFFFu : 0u;
                } else {
                    for (int i = 0; i < NT / 8; ++i) most = max(most, s_most[(c >> shift) * (NT / 8) + i]);
                }
                if (bound < LP_KEY_LOW || most > bound) again(v0 + c * CHUNK);
            }
            if (head > 0 || tail < a.V) {
                if (edge >= 0) add(lp_key(Vec::value(xr[edge])), edge);
                __syncthreads();
                rank_list(s_list, s_n);
            }
        }
    }

    // ---- the block's (max, l, S), and l - 1 where that is small
    float above = 0.0f;
    {
        float M = m;
#pragma unroll
        for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
        if (lane == 0) s_red[0][warp] = M;
        __syncthreads();
        M = s_red[0][0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) M = fmaxf(M, s_red[0][w]);
        float f = 1.0f, d = 0.0f;
        if (m != -INFINITY || l != 0.0f) {           // l without a maximum: a NaN
            d = m == -INFINITY ? 0.0f : diff(m, M);
            f = lp_exp2(d * scale2);
        }
        float ls = l * f, ss = l != 0.0f ? f * (S + l * d) : 0.0f;
        if (f == 0.0f && l == l) ls = ss = 0.0f;     // d may be -inf
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            ls += __shfl_xor_sync(0xFFFFFFFFu, ls, o);
            ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        }
        if (lane == 0) {
            s_red[1][warp] = ls;
            s_red[2][warp] = ss;
        }
        __syncthreads();
        float sum = 0.0f, sum_S = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            sum += s_red[1][w];
            sum_S += s_red[2][w];
        }
        if (sum < LP_SURE && M > -INFINITY) {          // the same for all threads
            float part = m == M ? 0.0f : l * f;
            int count = 0;
            uint32_t owners = __ballot_sync(0xFFFFFFFFu, m == M);
#pragma unroll 1
            for (; owners; owners &= owners - 1) {
                const int of = __ffs((int)owners) - 1;
                const int its_edge = __shfl_sync(0xFFFFFFFFu, edge, of);
                auto take = [&](float x) {
                    if (x == M) ++count;
                    else part += lp_exp2(diff(x, M) * scale2);
                };
                if (lane == 0 && its_edge >= 0) take(Vec::value(xr[its_edge]));
#pragma unroll 1
                for (int i = lane; i < chunks * U; i += 3 * 32) {
                    uint4 x[3];
#pragma unroll
                    for (int f = 0; f < 3; ++f) {
                        const int at = v0 + (i + f * 32) * NT + warp * 32 + of;
                        x[f].x = x[f].y = x[f].z = x[f].w = F32 ? 0xFF800000u : 0xFF80FF80u;
                        if (i + f * 32 < chunks * U && at < v1) x[f] = xv[at];
                    }
#pragma unroll
                    for (int f = 0; f < 3; ++f)
#pragma unroll
                        for (int e = 0; e < E; ++e) take(Vec::get(x[f], e));
                }
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                part += __shfl_xor_sync(0xFFFFFFFFu, part, o);
                count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
            }
            __syncthreads();             // the sums have been read
            if (lane == 0) {
                s_red[0][warp] = part;
                s_red[1][warp] = (float)count;
            }
            __syncthreads();
            float times = -1.0f;
            for (int w = 0; w < WARPS; ++w) {
                above += s_red[0][w];
                times += s_red[1][w];
            }
            above += times;              // 0, but for several maxima
        }
        m = M;
        l = sum;
        S = sum_S;
    }

    // ---- the cluster's: the others hand their sums and their k best to rank 0, which joins them in rank order
    if (cluster > 1) {
        if (rank) {
            if (TOP && tid < k) {
                const unsigned long long x = s_kept[which][tid];
                const uint32_t to = map_to_cta(smem_u32(s_in + (rank - 1) * k + tid), 0);
                st_cluster(to, (uint32_t)x);
                st_cluster(to + 4, (uint32_t)(x >> 32));
            }
            if (tid < 4) st_cluster(map_to_cta(smem_u32(&s_part[rank][tid]), 0), __float_as_uint(tid == 0 ? m : tid == 1 ? l : tid == 2 ? S : above));
        } else if (tid < 4) {
            s_part[0][tid] = tid == 0 ? m : tid == 1 ? l : tid == 2 ? S : above;
        }
        __syncwarp();
        cluster_sync_all();
        if (rank) return;
        m = -INFINITY;
        for (int c = 0; c < cluster; ++c) m = fmaxf(m, s_part[c][0]);
        l = S = 0.0f;
        above = 0.0f;
        for (int c = 0; c < cluster; ++c) {
            const float pl = s_part[c][1];
            if (pl == 0.0f) continue;
            const float d = s_part[c][0] == -INFINITY ? 0.0f : diff(s_part[c][0], m), f = lp_exp2(d * scale2);
            if (f == 0.0f && pl == pl) continue;
            l += pl * f;
            S += f * (s_part[c][2] + pl * d);
            above += s_part[c][0] == m ? s_part[c][3] : pl * f;      // (two blocks with the maximum: l is 2 at least)
        }
        if (TOP) rank_list(s_in, (cluster - 1) * k);
    }
    const float ln = l < LP_SURE ? log1pf(above) : logf(l), nan = __uint_as_float(0x7FC00000u);
    const bool empty = l == 0.0f;        // no logit above -inf
    const bool bad = m == INFINITY;
    auto logprob = [&](float x) { return bad ? nan : empty ? -INFINITY : 2.0f * rate * (0.5f * UNIT * x - 0.5f * UNIT * m) - ln; };      // (halves: x - m may pass the range)
    if (tid == 0) {
        if (a.lse) a.lse[row] = bad ? nan : empty ? -INFINITY : a.scale * m + ln;
        if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.0f : ln - rate * S / l;
    }
    for (int i = tid; i < a.n_ids; i += NT) {
        const int id = a.ids[row * a.ld_ids + i];
        a.logprob[row * a.n_ids + i] = id >= 0 && id < a.V ? logprob(Vec::value(xr[id])) : -INFINITY;
    }
    if (TOP) {
        for (int i = tid; i < k; i += NT) {
            const unsigned long long c = s_kept[which][i];
            const bool there = c != 0;
            a.top_ids[row * k + i] = there ? (int)~(uint32_t)c : -1;
            a.top_logprob[row * k + i] = there ? logprob(lp_value((uint32_t)(c >> 32))) : -INFINITY;
        }
    }
}

template <bool F32, bool TOP, int NT, bool SMALL = false>
static cudaError_t launch_logprobs_t(const LogprobArgs& a, int cluster, cudaStream_t st) {
    static PerDevice pd;
    constexpr int RING = LP_STAGES * NT * LP_VECS * 16;
    if (cudaError_t e = opt_in_shared_memory(pd, token_logprobs_kernel<F32, TOP, NT, SMALL>, RING)) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.T * cluster));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = RING;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<F32, TOP, NT, SMALL>, a, cluster);
}
template <bool F32, bool TOP>
static cudaError_t launch_logprobs(const LogprobArgs& a, int num_sms, cudaStream_t st) {
    if (a.scale < 1e-20f) return launch_logprobs_t<F32, TOP, 256, true>(a, 1, st);
    // Short rows, many of them: blocks of two warps, of which 16 are on an SM at a time, 11 with alternatives (shared memory).
    if ((int64_t)a.V * (F32 ? 4 : 2) <= LP_SHORT_BYTES) return launch_logprobs_t<F32, TOP, 64>(a, 1, st);
    // A cluster where the rows alone do not fill the machine, as long as every block of it has a chunk's work.
    const int64_t chunk = 256ll * LP_VECS * (F32 ? 4 : 8);
    int cluster = 1;
    while (cluster < LP_MAX_CLUSTER && (int64_t)a.T * cluster * 2 <= 3 * num_sms && (int64_t)a.V > chunk / 2 * cluster) cluster *= 2;
    return launch_logprobs_t<F32, TOP, 256>(a, cluster, st);
}

cudaError_t launch_token_logprobs(const LogprobArgs& a, bool f32, int num_sms, cudaStream_t st) {
    if (a.k) return f32 ? launch_logprobs<true, true>(a, num_sms, st) : launch_logprobs<false, true>(a, num_sms, st);
    return f32 ? launch_logprobs<true, false>(a, num_sms, st) : launch_logprobs<false, false>(a, num_sms, st);
}

}  // namespace osc
