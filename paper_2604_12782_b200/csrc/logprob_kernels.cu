// Log probabilities of given tokens, log-sum-exp, entropy and the best alternatives of every row of logits, in one pass.
//
//   d_j = x_j - max x,  l = sum_j exp(scale d_j),  S = sum_j d_j exp(scale d_j)
//   lse = scale max x + ln l,   log p_j = scale d_j - ln l,   entropy = ln l - scale S / l
//
// ln l and -S are never negative, so nothing cancels where a row is sure of one token.  A thread keeps its own (max, l, S) and joins a
// chunk of 16-byte vectors at a time: the chunk's maximum first, one correction of (l, S) if it is a new one, then the chunk's terms
// (l' = l f, S' = f (S + l (m - m')), f = exp(scale (m - m'))).  A row is one block's, or with few rows a cluster's, whose blocks take
// consecutive parts and are joined through distributed shared memory, so there is one launch and no workspace.
//
// Alternatives: the order is value, then lower index, as one key: the value's bits made monotone (NaN below -inf) and the index.  The chunk is in
// registers, and a thread's largest value is known from the maximum above.  First chunk: the k-th largest of the threads' largest values bounds
// the k-th best value of the row from below, and few other values pass it (with 256 threads and k = 20 less than one more), so the values
// at or above it go to a list in shared memory.  Later chunks: only values above the bound, a handful a chunk; a chunk without any costs one
// barrier that counts.  Where too many values pass (equal logits, rows in rising order) the chunk's best are taken one by one instead, k rounds of a
// maximum over the block.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"

namespace osc {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_VECS = 8;               // 16-byte vectors of a chunk, per thread
constexpr int LP_MAX_TOP = 32;
constexpr int LP_LIST = 1024;            // candidates that wait to be ranked
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
template <bool F32, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 3) token_logprobs_kernel(const LogprobArgs a, int cluster) {
    using Vec = LpVec<F32>;
    constexpr int E = Vec::E, U = LP_VECS;
    __shared__ unsigned long long s_list[TOP ? LP_LIST + LP_MAX_TOP : 1];    // candidates, the ranked ones first
    __shared__ unsigned long long s_best[TOP ? LP_MAX_TOP : 1];
    __shared__ uint32_t s_key[TOP ? LP_THREADS : 1];
    __shared__ unsigned long long s_warp[LP_WARPS];
    __shared__ float s_red[3][LP_WARPS];
    __shared__ float s_part[3];                      // (max, l, S) of the block
    __shared__ int s_n;
    __shared__ uint32_t s_bound;
    grid_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = cluster > 1 ? (int)cluster_ctarank() : 0;
    const int64_t row = blockIdx.x / cluster;
    const float scale2 = a.scale * 1.44269504088896341f;
    const int k = TOP ? a.k : 0;
    if (TOP && tid == 0) s_n = 0;
    grid_dependency_wait();

    // Rows begin at any element: vectors are counted from the 16-byte boundary at or before the row, `lead` elements of the first one are not the row's.
    const typename Vec::Elem* xr = static_cast<const typename Vec::Elem*>(a.x) + row * a.ld;
    const int lead = (int)((reinterpret_cast<uintptr_t>(xr) & 15u) / sizeof(typename Vec::Elem));
    const uint4* xv = reinterpret_cast<const uint4*>(xr - lead);
    const int nvec = (int)(((int64_t)lead + a.V + E - 1) / E);
    const int v0 = (int)((int64_t)nvec * rank / cluster), v1 = (int)((int64_t)nvec * (rank + 1) / cluster);
    const int full0 = lead ? 1 : 0, full1 = (int)(((int64_t)lead + a.V) / E);      // vectors [full0, full1) are the row's as a whole

    float m = -INFINITY, l = 0.0f, S = 0.0f;
    uint32_t bound = 0;          // values above it are candidates
    bool bounded = false;
    if (TOP) __syncthreads();

    // Ranks the candidates and keeps the k best, in order; `bound` is then the last one's key.
    auto rank_list = [&]() {
        __syncthreads();
        const int n = s_n;
        for (int i = tid; i < n; i += LP_THREADS) {
            const unsigned long long mine = s_list[i];
            int better = 0;
            for (int j = 0; j < n; ++j) better += s_list[j] > mine;
            if (better < k) s_best[better] = mine;
        }
        __syncthreads();
        const int kept = min(n, k);
        if (tid < kept) s_list[tid] = s_best[tid];
        if (tid == 0) s_n = kept;
        __syncthreads();
        if (kept == k) bound = (uint32_t)(s_list[k - 1] >> 32);
    };

#pragma unroll 1
    for (int base = v0; base < v1; base += LP_THREADS * U) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * LP_THREADS + tid;
            if (i >= full0 && i < full1 && i < v1) {
                v[u] = __ldcs(xv + i);
            } else {
                // the row's first or last vector, of which some elements are not the row's, or none at all: those read as -inf
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = F32 ? 0xFF800000u : 0xFF80FF80u;
                if (i < v1) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int j = i * E + e - lead;
                        if (j >= 0 && j < a.V) {
                            if (F32) w[e & 3] = __float_as_uint(Vec::value(xr[j]));
                            else {
                                const uint32_t b = __float_as_uint(Vec::value(xr[j]));
                                w[e / 2 & 3] = e & 1 ? (w[e / 2 & 3] & 0xFFFFu) | b : (w[e / 2 & 3] & 0xFFFF0000u) | b >> 16;
                            }
                        }
                    }
                }
                v[u] = make_uint4(w[0], w[1], w[2], w[3]);
            }
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
#pragma unroll
                for (int e = 0; e < 4; ++e) t = __hmax2(t, *reinterpret_cast<const __nv_bfloat162*>(&w[e]));
            }
            top = fmaxf(__low2float(t), __high2float(t));
        }
        // ---- (max, l, S)
        if (top > m) {
            if (m > -INFINITY) {
                const float d = m - top, f = lp_exp2(d * scale2);
                S = f == 0.0f ? 0.0f : f * (S + l * d);      // d may be -inf
                l *= f;
            }
            m = top;
        }
        {
            // A thread without a value above -inf has nothing to add; but a NaN has to reach the sums.
            const float ref = m == -INFINITY ? 0.0f : -m;
            const uint64_t ref2 = pack2(ref, ref), sc2 = pack2(scale2, scale2);
            uint64_t lc = 0, sc = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (base + u * LP_THREADS + tid >= v1) break;
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
            float sum = s0 + s1;
            if (sum != sum) {        // 0 * -inf: -inf among the logits (or a NaN, or +inf, which l shows)
                sum = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float d = Vec::get(v[u], e) + ref, p = lp_exp2(d * scale2);
                        sum += p == 0.0f ? 0.0f : p * d;
                    }
            }
            l += l0 + l1;
            S += sum;
        }
        // ---- candidates
        if (TOP) {
            // a NaN is a value too: a thread that holds nothing else has it as its largest
            uint32_t best = lp_key(top);
            const bool any = base + tid < v1;
            if (top == -INFINITY) {
                best = 0;
                if (any) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const int j = (base + u * LP_THREADS + tid) * E + e - lead;
                            if (base + u * LP_THREADS + tid < v1 && j >= 0 && j < a.V) best = max(best, lp_key(Vec::get(v[u], e)));
                        }
                }
            }
            const int before = s_n;
            uint32_t raised = 0;
            bool add;
            if (!bounded) {
                // k-th largest of the threads' largest values; ties by the thread
                s_key[tid] = best;
                __syncthreads();
                int better = 0;
#pragma unroll 8
                for (int j = 0; j < LP_THREADS; ++j) better += s_key[j] > best || (s_key[j] == best && j < tid);
                if (better == k - 1) s_bound = best;
                __syncthreads();
                raised = s_bound;
                bound = raised ? raised - 1 : 0;     // values at the bound are candidates themselves
                add = best > bound;
                bounded = true;
            } else {
                if (!__syncthreads_or(best > bound)) continue;
                add = best > bound;
            }
            if (add) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const uint32_t key = lp_key(Vec::get(v[u], e));
                        if (key > bound) {
                            const int i = base + u * LP_THREADS + tid, j = i * E + e - lead;
                            if (i < v1 && j >= 0 && j < a.V) {
                                const int at = atomicAdd(&s_n, 1);
                                if (at < LP_LIST) s_list[at] = lp_rank(key, j);
                            }
                        }
                    }
            }
            if (raised) bound = raised;          // of the chunks behind this one only values above it count: indices rise
            __syncthreads();
            if (s_n > LP_LIST) {
                // too many: the chunk's best one by one
                __syncthreads();
                if (tid == 0) s_n = before;
                bound = 0;
                rank_list();
                unsigned long long last = ~0ull;
#pragma unroll 1
                for (int i = 0; i < k; ++i) {
                    unsigned long long mine = 0;
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const int q = base + u * LP_THREADS + tid, j = q * E + e - lead;
                            if (q < v1 && j >= 0 && j < a.V) {
                                const unsigned long long c = lp_rank(lp_key(Vec::get(v[u], e)), j);
                                if (c < last && c > mine) mine = c;
                            }
                        }
#pragma unroll
                    for (int o = 16; o; o >>= 1) mine = max(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, o));
                    if (lane == 0) s_warp[warp] = mine;
                    __syncthreads();
                    unsigned long long best_of = s_warp[0];
#pragma unroll
                    for (int w = 1; w < LP_WARPS; ++w) best_of = max(best_of, s_warp[w]);
                    __syncthreads();
                    last = best_of;
                    if ((uint32_t)(last >> 32) <= bound) break;      // 0, or no better than the k of the chunks before
                    if (tid == 0) s_list[s_n++] = last;
                }
                rank_list();
            } else if (s_n > LP_LIST / 2) {
                rank_list();
            }
            __syncthreads();
        }
    }

    // ---- the block's (max, l, S)
    {
        float M = m;
#pragma unroll
        for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
        if (lane == 0) s_red[0][warp] = M;
        __syncthreads();
        M = s_red[0][0];
#pragma unroll
        for (int w = 1; w < LP_WARPS; ++w) M = fmaxf(M, s_red[0][w]);
        float f = 1.0f, d = 0.0f;
        if (m != -INFINITY || l != 0.0f) {           // l without a maximum: a NaN
            d = m == -INFINITY ? 0.0f : m - M;
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
        m = M;
        l = S = 0.0f;
#pragma unroll
        for (int w = 0; w < LP_WARPS; ++w) {
            l += s_red[1][w];
            S += s_red[2][w];
        }
        if (tid == 0) {
            s_part[0] = m;
            s_part[1] = l;
            s_part[2] = S;
        }
    }
    if (TOP) rank_list();

    // ---- the cluster's: every block joins the sums in rank order, rank 0 the candidates and the rest
    if (cluster > 1) {
        cluster_sync_all();
        if (rank == 0) {
            const uint32_t part = smem_u32(s_part), list = smem_u32(s_list), count = smem_u32(&s_n);
            auto ld32 = [](uint32_t addr) {
                uint32_t r;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(r) : "r"(addr) : "memory");
                return r;
            };
            float pm[LP_MAX_CLUSTER], pl[LP_MAX_CLUSTER], ps[LP_MAX_CLUSTER];
            m = -INFINITY;
#pragma unroll
            for (int c = 0; c < LP_MAX_CLUSTER; ++c)
                if (c < cluster) {
                    const uint32_t p = map_to_cta(part, c);
                    pm[c] = __uint_as_float(ld32(p));
                    pl[c] = __uint_as_float(ld32(p + 4));
                    ps[c] = __uint_as_float(ld32(p + 8));
                    m = fmaxf(m, pm[c]);
                }
            l = S = 0.0f;
#pragma unroll
            for (int c = 0; c < LP_MAX_CLUSTER; ++c)
                if (c < cluster && pl[c] != 0.0f) {
                    const float d = pm[c] == -INFINITY ? 0.0f : pm[c] - m, f = lp_exp2(d * scale2);
                    if (f == 0.0f && pl[c] == pl[c]) continue;
                    l += pl[c] * f;
                    S += f * (ps[c] + pl[c] * d);
                }
            if (TOP) {
                // the others' lists behind this block's: at most 8 * 32 candidates
                for (int c = 1; c < cluster; ++c) {
                    const int n = (int)ld32(map_to_cta(count, c)), at = s_n;
                    __syncthreads();
                    if (tid < n) {
                        const uint32_t p = map_to_cta(list, c) + tid * 8;
                        s_list[at + tid] = (unsigned long long)ld32(p + 4) << 32 | ld32(p);
                    }
                    if (tid == 0) s_n = at + n;
                    __syncthreads();
                }
                rank_list();
            }
        }
        cluster_sync_all();      // nobody leaves while its shared memory is read
        if (rank) return;
    }
    const float ln = logf(l), nan = __uint_as_float(0x7FC00000u);
    const bool empty = l == 0.0f;        // no logit above -inf
    const bool bad = m == INFINITY;
    auto logprob = [&](float x) { return bad ? nan : empty ? -INFINITY : a.scale * (x - m) - ln; };
    if (tid == 0) {
        if (a.lse) a.lse[row] = bad ? nan : empty ? -INFINITY : a.scale * m + ln;
        if (a.entropy) a.entropy[row] = bad ? nan : empty ? 0.0f : ln - a.scale * S / l;
    }
    for (int i = tid; i < a.n_ids; i += LP_THREADS) {
        const int id = a.ids[row * a.ld_ids + i];
        a.logprob[row * a.n_ids + i] = id >= 0 && id < a.V ? logprob(Vec::value(xr[id])) : -INFINITY;
    }
    if (TOP) {
        for (int i = tid; i < k; i += LP_THREADS) {
            const bool there = i < s_n;
            const unsigned long long c = s_list[there ? i : 0];
            a.top_ids[row * k + i] = there ? (int)~(uint32_t)c : -1;
            a.top_logprob[row * k + i] = there ? logprob(lp_value((uint32_t)(c >> 32))) : -INFINITY;
        }
    }
}

template <bool F32, bool TOP>
static cudaError_t launch_logprobs_t(const LogprobArgs& a, int cluster, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.T * cluster));
    cfg.blockDim = dim3(LP_THREADS);
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
    return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<F32, TOP>, a, cluster);
}

cudaError_t launch_token_logprobs(const LogprobArgs& a, bool f32, int num_sms, cudaStream_t st) {
    // A cluster where the rows alone do not fill the machine, as long as every block of it has a chunk's work.
    const int64_t chunk = (int64_t)LP_THREADS * LP_VECS * (f32 ? 4 : 8);
    int cluster = 1;
    while (cluster < LP_MAX_CLUSTER && (int64_t)a.T * cluster * 2 <= 6 * num_sms && (int64_t)a.V > chunk / 2 * cluster) cluster *= 2;
    if (a.k) return f32 ? launch_logprobs_t<true, true>(a, cluster, st) : launch_logprobs_t<false, true>(a, cluster, st);
    return f32 ? launch_logprobs_t<true, false>(a, cluster, st) : launch_logprobs_t<false, false>(a, cluster, st);
}

}  // namespace osc
