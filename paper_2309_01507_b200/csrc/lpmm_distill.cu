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

// One cluster of CTAs per row of logits, each CTA a slice of whole 16-byte vectors of it, which it holds in shared memory: the
// row is read from HBM once, and the gradient written once. Every thread copies, reduces and writes the same vectors, so that
// only the listed entries, which are taken out of the slice (set to -infinity), need barriers.
template <typename T, int THREADS, bool GRAD>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) distill_kernel(const DistillArgs a, const int cluster, const int slice_vecs) {
    using Bits = typename Row<T>::Bits;
    constexpr int VE = Row<T>::n, WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    uint4* const vec = reinterpret_cast<uint4*>(smem);
    Bits* const elem = reinterpret_cast<Bits*>(smem);
    int* const ids = reinterpret_cast<int*>(vec + slice_vecs);   // K ids, -1: no entry
    float* const lq = reinterpret_cast<float*>(ids + a.top);     // logarithms of the teacher's probabilities (see log_t)
    float* const zk = lq + a.top;                                // the student's logits at the ids of this slice
    __shared__ float part[WARPS][P_COUNT], loss_part[WARPS], teacher[2];
    __shared__ float ranks[kMaxCluster][P_COUNT], loss_ranks[kMaxCluster];
    const int K = a.top, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const float c = a.inv_tau * kLog2e;
    const bool tail = a.teacher_lse != nullptr;
    if (cluster > 1) cluster_barrier();       // every CTA is there before another stores into its shared memory

    for (int64_t t = blockIdx.x / cluster; t < a.tokens; t += gridDim.x / cluster) {
        const float w = a.weights ? a.weights[t] : 1.0f;
        const T* const z = static_cast<const T*>(a.logits) + t * a.logits_stride;
        T* const g = GRAD ? static_cast<T*>(a.grad) + t * a.grad_stride : nullptr;
        // The row's vectors start at the 16-byte boundary at or below its first element; this CTA holds [v0, v1).
        const int off = (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T)), V = (int)a.vocab;
        const int nvec = (off + V + VE - 1) / VE;
        const int v0 = (int)((int64_t)nvec * rank / cluster), v1 = (int)((int64_t)nvec * (rank + 1) / cluster);
        const int j0 = max(v0 * VE - off, 0), j1 = min(v1 * VE - off, V);     // its elements
        if (w == 0.0f) {
            if (rank == 0 && tid == 0) a.loss[t] = 0.0f;
            if constexpr (GRAD) for (int j = j0 + tid; j < j1; j += THREADS) g[j] = from_f32<T>(0.0f);
            continue;
        }
        for (int v = v0 + tid; v < v1; v += THREADS) {
            const int j = v * VE - off;
            if (j >= 0 && j + VE <= V) {
                copy16(vec + (v - v0), z + j);
            } else {
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    elem[(v - v0) * VE + i] = j + i >= 0 && j + i < V ? reinterpret_cast<const Bits*>(z)[j + i] : Row<T>::minus_inf;
            }
        }
        // Meanwhile one warp takes the teacher's entries.
        if (warp == 0) {
            float tmax = -INFINITY, st = 0.0f;
            for (int k = lane; k < K; k += 32) {
                const int64_t id = a.ids64 ? static_cast<const int64_t*>(a.ids)[t * K + k] : static_cast<const int32_t*>(a.ids)[t * K + k];
                const bool ok = id >= 0 && id < V;
                const float tl = ok ? load_f32(a.top_logits, a.top_dtype, t * K + k) : -INFINITY;
                ids[k] = ok ? (int)id : -1;
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
                st += expf(l);
            }
            st = warp_sum(st);
            if (lane == 0) {
                teacher[0] = st;
                teacher[1] = tail || !(st > 0.0f) ? 0.0f : logf(st);
            }
        }
        copies_landed();
        __syncthreads();
        const float s_t = teacher[0], log_t = teacher[1];
        // The listed entries of this slice leave it. An entry first puts its number into its element: where it then finds
        // another one, an id is listed twice.
        int twice = 0;
        for (int k = tid; k < K; k += THREADS) {
            const int id = ids[k], e = id + off - v0 * VE;
            if (id >= j0 && id < j1) zk[k] = to_f32(reinterpret_cast<const T*>(elem)[e]);
        }
        __syncthreads();
        for (int k = tid; k < K; k += THREADS) {
            const int id = ids[k];
            if (id >= j0 && id < j1) elem[id + off - v0 * VE] = (Bits)k;
        }
        __syncthreads();
        for (int k = tid; k < K; k += THREADS) {
            const int id = ids[k];
            if (id >= j0 && id < j1) twice |= elem[id + off - v0 * VE] != (Bits)k;
        }
        twice = __syncthreads_or(twice);
        float m_top = -INFINITY, s_top = 0.0f, n_top = 0.0f;
        for (int k = tid; k < K; k += THREADS) {
            const int id = ids[k];
            if (id >= j0 && id < j1) {
                elem[id + off - v0 * VE] = Row<T>::minus_inf;
                m_top = fmaxf(m_top, zk[k]);
            }
        }
        __syncthreads();
        if (warp * 32 < K) {
            m_top = warp_max1(m_top);
            for (int k = tid; k < K; k += THREADS) {
                const int id = ids[k];
                if (id < j0 || id >= j1) continue;
                bool first = true;       // every id counts once
                if (twice) for (int i = 0; i < k; ++i) first &= ids[i] != id;
                if (first) {
                    s_top += ex2((zk[k] - finite_ref(m_top)) * c);
                    n_top += 1.0f;
                }
            }
            s_top = warp_sum(s_top);
            n_top = warp_sum(n_top);
        }
        VecMax<T> vm;
#pragma unroll 4
        for (int v = tid; v < v1 - v0; v += THREADS) vm.add(vec[v]);
        float m_rest = warp_max1(vm.value()), s_rest = 0.0f;
        {
            const float ref = finite_ref(m_rest);
            const float2 neg = splat(-ref), c2 = splat(c);
            float2 sum = splat(0.0f);
#pragma unroll 2
            for (int v = tid; v < v1 - v0; v += THREADS) {
                float2 x[VE / 2];
                to_pairs<T>(vec[v], x);
#pragma unroll
                for (int i = 0; i < VE / 2; ++i) {
                    const float2 y = mul2_rn(add2_rn(x[i], neg), c2);
                    sum = add2_rn(sum, make_float2(ex2(y.x), ex2(y.y)));
                }
            }
            s_rest = warp_sum(sum.x + sum.y);
        }
        if (lane == 0) {
            part[warp][P_MREST] = m_rest; part[warp][P_SREST] = s_rest;
            part[warp][P_MTOP] = m_top; part[warp][P_STOP] = s_top; part[warp][P_NTOP] = n_top;
        }
        __syncthreads();
        {
            const bool in = lane < WARPS;
            float2 r = join_lanes(in ? part[lane][P_MREST] : -INFINITY, in ? part[lane][P_SREST] : 0.0f, c);
            m_rest = r.x; s_rest = r.y;
            r = join_lanes(in ? part[lane][P_MTOP] : -INFINITY, in ? part[lane][P_STOP] : 0.0f, c);
            m_top = r.x; s_top = r.y;
            n_top = warp_sum(in ? part[lane][P_NTOP] : 0.0f);
        }
        if (cluster > 1) {
            if (tid < cluster) {
                float* const mine = ranks[rank];
                store_at(mine + P_MREST, tid, m_rest); store_at(mine + P_SREST, tid, s_rest);
                store_at(mine + P_MTOP, tid, m_top); store_at(mine + P_STOP, tid, s_top); store_at(mine + P_NTOP, tid, n_top);
            }
            cluster_barrier();
            const bool in = lane < cluster;
            const float* const theirs = ranks[in ? lane : 0];
            float2 r = join_lanes(in ? theirs[P_MREST] : -INFINITY, in ? theirs[P_SREST] : 0.0f, c);
            m_rest = r.x; s_rest = r.y;
            r = join_lanes(in ? theirs[P_MTOP] : -INFINITY, in ? theirs[P_STOP] : 0.0f, c);
            m_top = r.x; s_top = r.y;
            n_top = warp_sum(in ? theirs[P_NTOP] : 0.0f);
        }
        const float m = finite_ref(fmaxf(m_rest, m_top));
        const float f_rest = ex2((m_rest - m) * c);                    // 0 when nothing is left out
        const float s = __fmaf_rn(s_rest, f_rest, s_top * ex2((m_top - m) * c));
        const float log_s = logf(s), inv_s = s > 0.0f || s != s ? 1.0f / s : 0.0f;
        const float q_rest = tail && n_top < (float)V ? fmaxf(1.0f - s_t, 0.0f) : 0.0f;
        const float Q = tail ? s_t + q_rest : (s_t > 0.0f || s_t != s_t) ? 1.0f : 0.0f;
        const float scale = w * a.inv_tau;
        if (warp * 32 < K) {
            float l = 0.0f;
            for (int k = tid; k < K; k += THREADS) {
                const int id = ids[k];
                if (id < j0 || id >= j1) continue;
                const float lqk = lq[k] - log_t, q = expf(lqk);
                if (q != 0.0f) l += q * (lqk - (zk[k] == -INFINITY && s == s ? -INFINITY : (zk[k] - m) * a.inv_tau - log_s));
            }
            l = warp_sum(l);
            if (lane == 0) loss_part[warp] = l;
        }
        if constexpr (GRAD) {
            // Left out: p_j (Q - q_rest / p_rest) with p_j = 2^(c (z_j - m_rest)) f_rest / s and p_rest = s_rest f_rest / s.
            const float coef = (Q * f_rest * inv_s - (s_rest > 0.0f ? q_rest / s_rest : 0.0f)) * scale;
            const float2 neg = splat(-finite_ref(m_rest)), c2 = splat(c), coef2 = splat(coef);
            if ((reinterpret_cast<uintptr_t>(g) - reinterpret_cast<uintptr_t>(z)) % 16 == 0) {
#pragma unroll 1
                for (int v = tid; v < v1 - v0; v += THREADS) {
                    float2 x[VE / 2];
                    to_pairs<T>(vec[v], x);
#pragma unroll
                    for (int i = 0; i < VE / 2; ++i) {
                        const float2 y = mul2_rn(add2_rn(x[i], neg), c2);
                        x[i] = mul2_rn(make_float2(ex2(y.x), ex2(y.y)), coef2);
                    }
                    const int j = (v0 + v) * VE - off;
                    if (j >= 0 && j + VE <= V) {
                        *reinterpret_cast<uint4*>(g + j) = from_pairs<T>(x);
                    } else {
#pragma unroll
                        for (int i = 0; i < VE; ++i)
                            if (j + i >= 0 && j + i < V) g[j + i] = from_f32<T>(i & 1 ? x[i / 2].y : x[i / 2].x);
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
                        const float zi = j + i >= j0 && j + i < j1 ? to_f32(reinterpret_cast<const T*>(elem)[j + i + off - v0 * VE]) : -INFINITY;
                        (i & 1 ? x[i / 2].y : x[i / 2].x) = ex2((zi + neg.x) * c) * coef;
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
            for (int k = tid; k < K; k += THREADS) {
                const int id = ids[k];
                if (id < j0 || id >= j1) continue;
                float q = 0.0f;
                if (twice) {
                    for (int i = 0; i < K; ++i) if (ids[i] == id) q += expf(lq[i] - log_t);
                } else {
                    q = expf(lq[k] - log_t);
                }
                g[id] = from_f32<T>((ex2((zk[k] - m) * c) * inv_s * Q - q) * scale);
            }
        }
        if (warp == 0) {
            float l = warp_sum(lane < WARPS && lane * 32 < K ? loss_part[lane] : 0.0f);
            if (cluster > 1) {
                if (lane == 0) store_at(&loss_ranks[rank], 0, l);
            } else if (lane == 0) {
                if (q_rest > 0.0f) l += q_rest * (logf(q_rest) - (s_rest > 0.0f ? (m_rest - m) * a.inv_tau + logf(s_rest) - log_s : -INFINITY));
                a.loss[t] = w * l;
            }
        }
        if (cluster > 1) {
            cluster_barrier();
            if (rank == 0 && tid == 0) {
                float l = 0.0f;
                for (int r = 0; r < cluster; ++r) l += loss_ranks[r];
                if (q_rest > 0.0f) l += q_rest * (logf(q_rest) - (s_rest > 0.0f ? (m_rest - m) * a.inv_tau + logf(s_rest) - log_s : -INFINITY));
                a.loss[t] = w * l;
            }
        } else {
            __syncthreads();
        }
    }
}

template <typename T, int THREADS, bool GRAD>
cudaError_t launch(const DistillArgs& a, int cluster, int slice_vecs, size_t bytes, cudaStream_t s) {
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
    e = cudaLaunchKernelEx(&cfg, kernel, a, cluster, slice_vecs);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, int logits_dtype, cudaStream_t s) {
    const int64_t es = logits_dtype == 0 ? 4 : 2;
    const int64_t row_vecs = a.vocab * es / 16 + 2;    // however the row is aligned
    // Slices of up to 64 KB, three of which an SM holds at a time; eight CTAs at most. Few rows are split further, until every
    // SM has a CTA or a slice is down to 8 KB.
    int cluster = 1;
    while (cluster < kMaxCluster && row_vecs > cluster * (int64_t)4096) cluster *= 2;
    while (cluster < kMaxCluster && a.tokens * cluster < 148 && row_vecs > cluster * (int64_t)1024) cluster *= 2;
    const int slice = (int)((row_vecs + cluster - 1) / cluster) + 1;
    const size_t bytes = (size_t)slice * 16 + (size_t)a.top * 12;
    return with_dtype(logits_dtype, [&](auto t) {
        using T = decltype(t);
        if (slice <= 1024) return a.grad ? launch<T, 128, true>(a, cluster, slice, bytes, s) : launch<T, 128, false>(a, cluster, slice, bytes, s);
        return a.grad ? launch<T, 512, true>(a, cluster, slice, bytes, s) : launch<T, 512, false>(a, cluster, slice, bytes, s);
    });
}

}  // namespace lpmm
