// Distillation from a teacher's top logits, loss and gradient in one launch, for sm_100a.
//
// For a row with logits z, temperature tau and K listed entries (id_k, t_k):
//   p = softmax(z / tau),  q_k = softmax(t / tau) over the listed entries, or exp(t_k / tau - lse) with the teacher's own
//   log-sum-exp, and then q_rest = 1 - sum q for the entries left out, p_rest = the sum of their p;
//   loss = w [ sum q_k (log q_k - log p_{id_k}) + q_rest (log q_rest - log p_rest) ],
//   d loss / d z_j = (w / tau) (p_j Q - sum_{k: id_k = j} q_k)    for a listed j,
//                    (w / tau) p_j (Q - q_rest / p_rest)          for one left out,  Q = sum q + q_rest.
// Powers are taken in base 2 of c (z_j - max z), c = log2(e) / tau: the difference first, so that logits masked with the type's
// lowest value cannot overflow. p_rest is summed over the entries left out themselves, relative to their own maximum, never
// taken as 1 - sum p: it keeps its precision, and its logarithm, when the student is sure of the listed entries.
#include <algorithm>

#include "lpmm_internal.h"
#include "lpmm_ops.cuh"

namespace lpmm {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_max1(float x) {   // one instruction on sm_100a; NaN loses, as with fmaxf
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_sum(float x) {
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}
// Stores v at `here`'s place in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ void store_at(float* here, uint32_t rank, float v) {
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_addr(here)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}

template <typename T> struct Row;   // a logits type: elements per 16 bytes, one element as bits, -infinity
template <> struct Row<float> { using Bits = uint32_t; static constexpr int n = 4; static constexpr Bits minus_inf = 0xff800000u; };
template <> struct Row<__nv_bfloat16> { using Bits = uint16_t; static constexpr int n = 8; static constexpr Bits minus_inf = 0xff80u; };
template <> struct Row<__half> { using Bits = uint16_t; static constexpr int n = 8; static constexpr Bits minus_inf = 0xfc00u; };

// The elements of a 16-byte vector as pairs of binary32.
template <typename T> __device__ __forceinline__ void to_pairs(uint4 q, float2 (&v)[Row<T>::n / 2]) {
    if constexpr (sizeof(T) == 4) {
        v[0] = make_float2(__uint_as_float(q.x), __uint_as_float(q.y));
        v[1] = make_float2(__uint_as_float(q.z), __uint_as_float(q.w));
    } else {
        v[0] = unpack_pair<T>(q.x); v[1] = unpack_pair<T>(q.y); v[2] = unpack_pair<T>(q.z); v[3] = unpack_pair<T>(q.w);
    }
}
template <typename T> __device__ __forceinline__ uint4 from_pairs(const float2 (&v)[Row<T>::n / 2]) {
    if constexpr (sizeof(T) == 4) {
        return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
    } else {
        return make_uint4(pack_pair<T>(v[0].x, v[0].y), pack_pair<T>(v[1].x, v[1].y), pack_pair<T>(v[2].x, v[2].y), pack_pair<T>(v[3].x, v[3].y));
    }
}
// Running maximum of vectors; 16-bit types compare two elements at a time in their own type.
template <typename T> struct VecMax {
    float m = -INFINITY;
    __device__ __forceinline__ void add(uint4 q) {
        m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(q.x)), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
    __device__ __forceinline__ float value() const { return m; }
};
template <typename P, typename T> struct PairMax {
    uint32_t m = (uint32_t)Row<T>::minus_inf * 0x10001u;
    __device__ __forceinline__ static uint32_t mx(uint32_t a, uint32_t b) {
        const P r = __hmax2(*reinterpret_cast<const P*>(&a), *reinterpret_cast<const P*>(&b));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    __device__ __forceinline__ void add(uint4 q) { m = mx(mx(m, mx(q.x, q.y)), mx(q.z, q.w)); }
    __device__ __forceinline__ float value() const { const float2 p = unpack_pair<T>(m); return fmaxf(p.x, p.y); }
};
template <> struct VecMax<__nv_bfloat16> : PairMax<__nv_bfloat162, __nv_bfloat16> {};
template <> struct VecMax<__half> : PairMax<__half2, __half> {};

// A class of a row's entries (those left out, or the listed ones): the maximum of its logits and the sum of the powers relative
// to it. Parts are joined by bringing them to the larger maximum; an empty part has maximum -infinity and sum 0.
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float2 join_lanes(float m, float s, float c) {
    const float M = warp_max1(m);
    return make_float2(M, warp_sum(s * ex2((m - finite_ref(M)) * c)));
}

enum { P_MREST, P_SREST, P_MTOP, P_STOP, P_NTOP, P_COUNT };   // what warps, and then CTAs of a cluster, exchange

// What one warp works out for a row and all others read.
struct RowResult {
    float ref, coef;           // left out: gradient = coef 2^(c (z - ref))
    float m, q_scale, scale;   // listed: q_scale 2^(c (z - m)) - q scale
};

// One cluster of CTAs per row of logits, each CTA a slice of whole 16-byte vectors of it, which it holds in shared memory: the
// row is read from HBM once, and the gradient written once. Every thread copies, reduces and writes the same vectors, so that
// only the listed entries, which are taken out of the slice (set to -infinity), need barriers. The first `entry_warps` warps
// take the listed entries, warp 0 the teacher and what is worked out once per row.
template <typename T, int THREADS, bool GRAD>
__global__ void __launch_bounds__(THREADS, 768 / THREADS) distill_kernel(const DistillArgs a, const int log_cluster, const int slice_vecs, const int entry_warps) {
    using Bits = typename Row<T>::Bits;
    constexpr int VE = Row<T>::n, WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    uint4* const vec = reinterpret_cast<uint4*>(smem);
    Bits* const elem = reinterpret_cast<Bits*>(smem);
    int* const slot = reinterpret_cast<int*>(vec + slice_vecs);   // K ids, later the element in the slice; -1: no entry here
    float* const lq = reinterpret_cast<float*>(slot + a.top);     // logarithms of the teacher's probabilities
    float* const zk = lq + a.top;                                 // the student's logits at the ids of this slice
    __shared__ float part[WARPS][P_COUNT], top_part[WARPS][2];
    __shared__ float ranks[kMaxCluster][P_COUNT + 2];
    __shared__ RowResult result;
    const int K = a.top, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, estride = entry_warps * 32;
    const int cluster = 1 << log_cluster, rank = log_cluster ? (int)cluster_rank() : 0;
    const float c = a.inv_tau * kLog2e;
    const bool tail = a.teacher_lse != nullptr, entries = warp < entry_warps;
    if (log_cluster) cluster_barrier();       // every CTA is there before another stores into its shared memory

    for (int64_t t = blockIdx.x >> log_cluster; t < a.tokens; t += gridDim.x >> log_cluster) {
        const float w = a.weights ? a.weights[t] : 1.0f;
        const T* const z = static_cast<const T*>(a.logits) + t * a.logits_stride;
        T* const g = GRAD ? static_cast<T*>(a.grad) + t * a.grad_stride : nullptr;
        // The row's vectors start at the 16-byte boundary at or below its first element; this CTA holds [v0, v1).
        const int off = (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T)), V = (int)a.vocab;
        const int nvec = (off + V + VE - 1) / VE;
        const int v0 = (nvec * rank) >> log_cluster, v1 = (nvec * (rank + 1)) >> log_cluster, nv = v1 - v0;
        const int e0 = v0 * VE - off;                                         // the entry in the slice's first element
        const int j0 = max(e0, 0), j1 = min(v1 * VE - off, V);                // its entries
        const int whole0 = e0 < 0 ? 1 : 0, whole1 = v1 * VE - off > V ? nv - 1 : nv;   // vectors that lie in the row entirely
        if (w == 0.0f) {
            if (rank == 0 && tid == 0) a.loss[t] = 0.0f;
            if constexpr (GRAD) for (int j = j0 + tid; j < j1; j += THREADS) g[j] = from_f32<T>(0.0f);
            continue;
        }
        {
            const uint4* const src = reinterpret_cast<const uint4*>(z + e0);
            for (int v = tid; v < nv; v += THREADS) {
                if (v >= whole0 && v < whole1) {
                    copy16(vec + v, src + v);
                } else {
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        const int j = e0 + v * VE + i;
                        elem[v * VE + i] = j >= 0 && j < V ? reinterpret_cast<const Bits*>(z)[j] : Row<T>::minus_inf;
                    }
                }
            }
        }
        // Meanwhile warp 0 takes the teacher's entries.
        float s_t = 0.0f;
        if (warp == 0) {
            float tmax = -INFINITY;
            for (int k = lane; k < K; k += 32) {
                const int64_t id = a.ids64 ? static_cast<const int64_t*>(a.ids)[t * K + k] : static_cast<const int32_t*>(a.ids)[t * K + k];
                const bool ok = id >= 0 && id < V;
                const float tl = ok ? load_f32(a.top_logits, a.top_dtype, t * K + k) : -INFINITY;
                slot[k] = ok && id >= j0 && id < j1 ? (int)id - e0 : -1;
                lq[k] = tl;
                tmax = fmaxf(tmax, tl);
            }
            tmax = finite_ref(warp_max1(tmax));
            const float lse = tail ? a.teacher_lse[t] : 0.0f;
            for (int k = lane; k < K; k += 32) {
                const float tl = lq[k];
                // -infinity stays: its products with the two parts of 1 / tau could cancel to NaN
                const float l = tl == -INFINITY ? tl : tail ? __fmaf_rn(tl, a.inv_tau, __fmaf_rn(tl, a.inv_tau_lo, -lse)) : (tl - tmax) * a.inv_tau;
                lq[k] = l;
                s_t += expf(l);
            }
            s_t = warp_sum(s_t);
            if (!tail && s_t > 0.0f) {
                const float log_t = logf(s_t);
                for (int k = lane; k < K; k += 32) lq[k] -= log_t;
            }
        }
        copies_landed();
        __syncthreads();
        // The listed entries of this slice leave it. An entry first puts its number into its element: where it then finds
        // another one, an id is listed twice.
        int twice = 0;
        if (entries) {
            const auto together = [&] { asm volatile("bar.sync 1, %0;" ::"r"(estride) : "memory"); };
            float m_top = -INFINITY, s_top = 0.0f, n_top = 0.0f;
            for (int k = tid; k < K; k += estride) {
                const int e = slot[k];
                if (e >= 0) m_top = fmaxf(m_top, zk[k] = to_f32(reinterpret_cast<const T*>(elem)[e]));
            }
            m_top = warp_max1(m_top);
            together();
            for (int k = tid; k < K; k += estride) if (const int e = slot[k]; e >= 0) elem[e] = (Bits)k;
            together();
            for (int k = tid; k < K; k += estride) if (const int e = slot[k]; e >= 0) twice |= elem[e] != (Bits)k;
            asm volatile("{\n.reg .pred p, q;\nsetp.ne.s32 p, %1, 0;\nbar.red.or.pred q, 1, %2, p;\nselp.s32 %0, 1, 0, q;\n}" : "=r"(twice) : "r"(twice), "r"(estride) : "memory");
            for (int k = tid; k < K; k += estride) {
                const int e = slot[k];
                if (e < 0) continue;
                elem[e] = Row<T>::minus_inf;
                bool first = true;       // every id counts once
                if (twice) for (int i = 0; i < k; ++i) first &= slot[i] != e;
                if (first) {
                    s_top += ex2((zk[k] - finite_ref(m_top)) * c);
                    n_top += 1.0f;
                }
            }
            s_top = warp_sum(s_top);
            n_top = warp_sum(n_top);
            if (lane == 0) { part[warp][P_MTOP] = m_top; part[warp][P_STOP] = s_top; part[warp][P_NTOP] = n_top; }
        }
        __syncthreads();
        {
            VecMax<T> vm;
#pragma unroll 4
            for (int v = tid; v < nv; v += THREADS) vm.add(vec[v]);
            const float m = warp_max1(vm.value());
            const float2 neg = splat(-finite_ref(m)), c2 = splat(c);
            float2 sum = splat(0.0f);
#pragma unroll 2
            for (int v = tid; v < nv; v += THREADS) {
                float2 x[VE / 2];
                to_pairs<T>(vec[v], x);
#pragma unroll
                for (int i = 0; i < VE / 2; ++i) {
                    const float2 y = mul2_rn(add2_rn(x[i], neg), c2);
                    sum = add2_rn(sum, make_float2(ex2(y.x), ex2(y.y)));
                }
            }
            const float s = warp_sum(sum.x + sum.y);
            if (lane == 0) { part[warp][P_MREST] = m; part[warp][P_SREST] = s; }
        }
        __syncthreads();
        float m = 0.0f, m_rest = 0.0f, s_rest = 0.0f, log_s = 0.0f, s = 0.0f, q_rest = 0.0f;
        if (warp == 0) {
            bool in = lane < WARPS;
            float2 rest = join_lanes(in ? part[lane][P_MREST] : -INFINITY, in ? part[lane][P_SREST] : 0.0f, c);
            in = lane < entry_warps;
            float2 top = join_lanes(in ? part[lane][P_MTOP] : -INFINITY, in ? part[lane][P_STOP] : 0.0f, c);
            float n_top = warp_sum(in ? part[lane][P_NTOP] : 0.0f);
            if (log_cluster) {
                if (lane < cluster) {
                    float* const mine = ranks[rank];
                    store_at(mine + P_MREST, lane, rest.x); store_at(mine + P_SREST, lane, rest.y);
                    store_at(mine + P_MTOP, lane, top.x); store_at(mine + P_STOP, lane, top.y); store_at(mine + P_NTOP, lane, n_top);
                }
            }
            part[0][P_MREST] = rest.x; part[0][P_SREST] = rest.y; part[0][P_MTOP] = top.x; part[0][P_STOP] = top.y; part[0][P_NTOP] = n_top;
        }
        if (log_cluster) cluster_barrier();
        if (warp == 0) {
            float2 rest, top;
            float n_top;
            if (log_cluster) {
                const bool in = lane < cluster;
                const float* const r = ranks[in ? lane : 0];
                rest = join_lanes(in ? r[P_MREST] : -INFINITY, in ? r[P_SREST] : 0.0f, c);
                top = join_lanes(in ? r[P_MTOP] : -INFINITY, in ? r[P_STOP] : 0.0f, c);
                n_top = warp_sum(in ? r[P_NTOP] : 0.0f);
            } else {
                __syncwarp();
                rest = make_float2(part[0][P_MREST], part[0][P_SREST]);
                top = make_float2(part[0][P_MTOP], part[0][P_STOP]);
                n_top = part[0][P_NTOP];
            }
            m_rest = rest.x; s_rest = rest.y;
            m = finite_ref(fmaxf(m_rest, top.x));
            const float f_rest = ex2((m_rest - m) * c);                    // 0 when nothing is left out
            s = __fmaf_rn(s_rest, f_rest, top.y * ex2((top.x - m) * c));
            const float inv_s = s > 0.0f || s != s ? 1.0f / s : 0.0f;
            log_s = logf(s);
            q_rest = tail && n_top < (float)V ? fmaxf(1.0f - s_t, 0.0f) : 0.0f;
            const float Q = tail ? s_t + q_rest : (s_t > 0.0f || s_t != s_t) ? 1.0f : 0.0f;
            const float scale = w * a.inv_tau;
            // Left out: p_j (Q - q_rest / p_rest) with p_j = 2^(c (z_j - m_rest)) f_rest / s and p_rest = s_rest f_rest / s.
            if (lane == 0) {
                result.ref = finite_ref(m_rest);
                result.coef = (Q * f_rest * inv_s - (s_rest > 0.0f ? q_rest / s_rest : 0.0f)) * scale;
                result.m = m;
                result.q_scale = Q * inv_s * scale;
                result.scale = scale;
                top_part[0][0] = log_s;
                top_part[0][1] = s;
            }
        }
        __syncthreads();
        const RowResult res = result;
        if (entries) {      // this slice's share of the loss
            const float log_all = top_part[0][0], all = top_part[0][1];
            float l = 0.0f;
            for (int k = tid; k < K; k += estride) {
                if (slot[k] < 0) continue;
                const float q = expf(lq[k]);
                if (q != 0.0f) l += q * (lq[k] - (zk[k] == -INFINITY && all == all ? -INFINITY : (zk[k] - res.m) * a.inv_tau - log_all));
            }
            l = warp_sum(l);
            if (lane == 0) part[warp][P_MTOP] = l;
        }
        if constexpr (GRAD) {
            const float2 neg = splat(-res.ref), c2 = splat(c), coef2 = splat(res.coef);
            if ((reinterpret_cast<uintptr_t>(g) - reinterpret_cast<uintptr_t>(z)) % 16 == 0) {
                uint4* const dst = reinterpret_cast<uint4*>(g + e0);
#pragma unroll 2
                for (int v = tid; v < nv; v += THREADS) {
                    float2 x[VE / 2];
                    to_pairs<T>(vec[v], x);
#pragma unroll
                    for (int i = 0; i < VE / 2; ++i) {
                        const float2 y = mul2_rn(add2_rn(x[i], neg), c2);
                        x[i] = mul2_rn(make_float2(ex2(y.x), ex2(y.y)), coef2);
                    }
                    if (v >= whole0 && v < whole1) {
                        dst[v] = from_pairs<T>(x);
                    } else {
#pragma unroll
                        for (int i = 0; i < VE; ++i) {
                            const int j = e0 + v * VE + i;
                            if (j >= 0 && j < V) g[j] = from_f32<T>(i & 1 ? x[i / 2].y : x[i / 2].x);
                        }
                    }
                }
            } else {
                // The gradient's rows are aligned otherwise than the logits': its own vectors, gathered element by element.
                const int goff = (int)(reinterpret_cast<uintptr_t>(g) % 16 / sizeof(T));
                const int u1 = (j1 + goff + VE - 1) / VE;
#pragma unroll 1
                for (int u = (j0 + goff) / VE + tid; u < u1; u += THREADS) {
                    const int j = u * VE - goff;
                    float2 x[VE / 2];
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        const float zi = j + i >= j0 && j + i < j1 ? to_f32(reinterpret_cast<const T*>(elem)[j + i - e0]) : -INFINITY;
                        (i & 1 ? x[i / 2].y : x[i / 2].x) = ex2((zi + neg.x) * c) * res.coef;
                    }
                    if (j >= j0 && j + VE <= j1) {
                        *reinterpret_cast<uint4*>(g + j) = from_pairs<T>(x);
                    } else {
#pragma unroll
                        for (int i = 0; i < VE; ++i)
                            if (j + i >= j0 && j + i < j1) g[j + i] = from_f32<T>(i & 1 ? x[i / 2].y : x[i / 2].x);
                    }
                }
            }
        }
        __syncthreads();        // the listed entries' gradients go over the slice's, and the warps' shares of the loss are there
        if constexpr (GRAD) {
            if (entries) {
                for (int k = tid; k < K; k += estride) {
                    const int e = slot[k];
                    if (e < 0) continue;
                    float q = 0.0f;
                    if (twice) {
                        for (int i = 0; i < K; ++i) if (slot[i] == e) q += expf(lq[i]);
                    } else {
                        q = expf(lq[k]);
                    }
                    g[e0 + e] = from_f32<T>(__fmaf_rn(ex2((zk[k] - res.m) * c), res.q_scale, -q * res.scale));
                }
            }
        }
        if (warp == 0) {
            float l = warp_sum(lane < entry_warps ? part[lane][P_MTOP] : 0.0f);
            if (log_cluster) {
                if (lane == 0) store_at(&ranks[rank][P_COUNT], 0, l);
            }
            if (rank == 0 && q_rest > 0.0f) s_t = q_rest * (logf(q_rest) - (s_rest > 0.0f ? (m_rest - m) * a.inv_tau + logf(s_rest) - log_s : -INFINITY));
            else s_t = 0.0f;
            if (!log_cluster && lane == 0) a.loss[t] = w * (l + s_t);
        }
        if (log_cluster) {
            cluster_barrier();
            if (rank == 0 && tid == 0) {
                float l = 0.0f;
                for (int r = 0; r < cluster; ++r) l += ranks[r][P_COUNT];
                a.loss[t] = w * (l + s_t);
            }
        } else {
            __syncthreads();
        }
    }
}

template <typename T, int THREADS, bool GRAD>
cudaError_t launch(const DistillArgs& a, int log_cluster, int slice_vecs, size_t bytes, cudaStream_t s) {
    const int cluster = 1 << log_cluster;
    auto kernel = distill_kernel<T, THREADS, GRAD>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    const int64_t rows = a.tokens < (1 << 24) ? a.tokens : 1 << 24;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kernel, a, log_cluster, slice_vecs, std::min(THREADS / 32, (a.top + 63) / 64));
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, int logits_dtype, cudaStream_t s) {
    const int64_t es = logits_dtype == 0 ? 4 : 2;
    const int64_t row_vecs = a.vocab * es / 16 + 2;    // however the row is aligned
    // Slices of up to 64 KB, three of which an SM holds at a time; eight CTAs at most. Few rows are split further, until every
    // SM has a CTA or a slice is down to 8 KB.
    int log_cluster = 0;
    while (log_cluster < 3 && row_vecs > (int64_t)4096 << log_cluster) ++log_cluster;
    while (log_cluster < 3 && a.tokens << log_cluster < 148 && row_vecs > (int64_t)1024 << log_cluster) ++log_cluster;
    const int slice = (int)((row_vecs + (1 << log_cluster) - 1) >> log_cluster) + 1;
    const size_t bytes = (size_t)slice * 16 + (size_t)a.top * 12;
    return with_dtype(logits_dtype, [&](auto t) {
        using T = decltype(t);
        if (slice <= 1024) return a.grad ? launch<T, 128, true>(a, log_cluster, slice, bytes, s) : launch<T, 128, false>(a, log_cluster, slice, bytes, s);
        return a.grad ? launch<T, 256, true>(a, log_cluster, slice, bytes, s) : launch<T, 256, false>(a, log_cluster, slice, bytes, s);
    });
}

}  // namespace lpmm
