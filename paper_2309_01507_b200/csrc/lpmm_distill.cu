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
constexpr int blocks_per_sm(int threads) { return threads == 256 ? 3 : 8; }

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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() { cluster_arrive(); cluster_wait(); }
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

// Where a CTA's slice of a row lies: whole 16-byte vectors from the boundary at or below the row's first element on.
template <typename T> struct Slice {
    const T* z;
    int nv, e0, j0, j1;       // vectors; the row's entry in the first element; the entries [j0, j1) that lie in the row
    int whole0, whole1;       // the vectors that do entirely
    __device__ __forceinline__ Slice(const DistillArgs& a, int64_t t, int rank, int log_cluster) {
        constexpr int VE = Row<T>::n;
        z = static_cast<const T*>(a.logits) + t * a.logits_stride;
        const int off = (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T)), V = (int)a.vocab;
        const int n = (off + V + VE - 1) / VE, v0 = (n * rank) >> log_cluster, v1 = (n * (rank + 1)) >> log_cluster;
        nv = v1 - v0;
        e0 = v0 * VE - off;
        j0 = max(e0, 0);
        j1 = min(v1 * VE - off, V);
        whole0 = e0 < 0 ? 1 : 0;
        whole1 = v1 * VE - off > V ? nv - 1 : nv;
    }
    // Starts the copy of vector v; -infinity where it reaches out of the row.
    __device__ __forceinline__ void fetch(uint4* vec, int v, int V) const {
        if (v >= whole0 && v < whole1) {
            copy16(vec + v, reinterpret_cast<const uint4*>(z + e0) + v);
        } else {
            using Bits = typename Row<T>::Bits;
#pragma unroll
            for (int i = 0; i < Row<T>::n; ++i) {
                const int j = e0 + v * Row<T>::n + i;
                reinterpret_cast<Bits*>(vec + v)[i] = j >= 0 && j < V ? reinterpret_cast<const Bits*>(z)[j] : Row<T>::minus_inf;
            }
        }
    }
};

// The first row from t on, in steps of `step`, that has a weight. weight_at() is asked 32 rows ahead, one per lane.
__device__ __forceinline__ float weight_ahead(const DistillArgs& a, int64_t t, int64_t step) {
    const int64_t i = t + (threadIdx.x & 31) * step;
    return i < a.tokens && a.weights ? a.weights[i] : 1.0f;
}
__device__ __forceinline__ int64_t live_row(const DistillArgs& a, int64_t t, int64_t step, float ahead) {
    for (;;) {
        const uint32_t live = __ballot_sync(0xffffffffu, ahead != 0.0f);
        if (live) return min(t + (__ffs(live) - 1) * step, a.tokens);
        t += 32 * step;
        ahead = weight_ahead(a, t, step);
    }
}

// Barriers: all warps of the CTA, when a row and its teacher's side are in shared memory; the workers alone, within a row.
template <int THREADS> __device__ __forceinline__ void row_ready() { asm volatile("bar.sync 0, %0;" ::"n"(THREADS + 32) : "memory"); }
template <int THREADS> __device__ __forceinline__ void workers_together() { asm volatile("bar.sync 2, %0;" ::"n"(THREADS) : "memory"); }

// One cluster of CTAs per row of logits, each CTA a slice of it, which it holds in shared memory: the row is read from HBM once,
// and the gradient written once. Each of the THREADS workers copies, reduces and writes the same vectors of every row, so that
// only the listed entries, which are taken out of the slice (set to -infinity), need barriers, and a worker fetches a vector
// of the next row as soon as it is done with this row's. The first `entry_warps` warps take the listed entries; one more warp
// prepares the teacher's side of the next row meanwhile.
template <typename T, int THREADS, bool GRAD>
__global__ void __launch_bounds__(THREADS + 32, blocks_per_sm(THREADS)) distill_kernel(const DistillArgs a, const int log_cluster, const int slice_vecs, const int entry_warps) {
    using Bits = typename Row<T>::Bits;
    constexpr int VE = Row<T>::n, WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    uint4* const vec = reinterpret_cast<uint4*>(smem);
    Bits* const elem = reinterpret_cast<Bits*>(smem);
    const int K = a.top;
    int* const slots = reinterpret_cast<int*>(vec + slice_vecs);   // 2 x K: the element in the slice; -1: no entry here
    float* const lqs = reinterpret_cast<float*>(slots + 2 * K);    // 2 x K: logarithms of the teacher's probabilities
    float* const zk = lqs + 2 * K;                                 // the student's logits at the slots
    __shared__ float part[WARPS][P_COUNT], loss_part[WARPS], teacher[2][2];
    __shared__ float ranks[kMaxCluster][P_COUNT + 1];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, estride = entry_warps * 32, V = (int)a.vocab;
    const int cluster = 1 << log_cluster, rank = log_cluster ? (int)cluster_rank() : 0;
    const float c = a.inv_tau * kLog2e;
    const bool tail = a.teacher_lse != nullptr, entries = warp < entry_warps;
    const int64_t step = gridDim.x >> log_cluster, first_row = blockIdx.x >> log_cluster;
    if (log_cluster) cluster_barrier();       // every CTA is there before another stores into its shared memory
    int64_t t = live_row(a, first_row, step, weight_ahead(a, first_row, step));
    int buf = 0;

    if (warp == WARPS) {                      // the teacher
        const auto prepare = [&](int64_t t, int buf) {
            int* const slot = slots + buf * K;
            float* const lq = lqs + buf * K;
            const float w = a.weights ? a.weights[t] : 1.0f, lse = tail ? a.teacher_lse[t] : 0.0f;
            const Slice<T> sl(a, t, rank, log_cluster);
            float tmax = -INFINITY, s_t = 0.0f;
            for (int k = lane; k < K; k += 32) {
                const int64_t id = a.ids64 ? static_cast<const int64_t*>(a.ids)[t * K + k] : static_cast<const int32_t*>(a.ids)[t * K + k];
                float tl = load_f32(a.top_logits, a.top_dtype, t * K + k);
                if (id < 0 || id >= V) tl = -INFINITY;
                slot[k] = id >= sl.j0 && id < sl.j1 ? (int)id - sl.e0 : -1;
                lq[k] = tl;
                tmax = fmaxf(tmax, tl);
            }
            tmax = finite_ref(warp_max1(tmax));
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
            if (lane == 0) { teacher[buf][0] = s_t; teacher[buf][1] = w; }
        };
        if (t < a.tokens) prepare(t, 0);
        while (t < a.tokens) {
            const float ahead = weight_ahead(a, t + step, step);
            row_ready<THREADS>();
            if (log_cluster) cluster_arrive();
            t = live_row(a, t + step, step, ahead);
            if (t < a.tokens) prepare(t, buf ^= 1);
            if (log_cluster) { cluster_wait(); cluster_barrier(); }
        }
        return;
    }

    if (t < a.tokens) {
        const Slice<T> sl(a, t, rank, log_cluster);
        for (int v = tid; v < sl.nv; v += THREADS) sl.fetch(vec, v, V);
    }
    if (a.weights) {                          // rows without a weight, while the first one arrives
        for (int64_t r = first_row; r < a.tokens; r += step) {
            if (a.weights[r] != 0.0f) continue;
            if (rank == 0 && tid == 0) a.loss[r] = 0.0f;
            if constexpr (GRAD) {
                T* const g = static_cast<T*>(a.grad) + r * a.grad_stride;
                const Slice<T> sl(a, r, rank, log_cluster);
                const int j0 = min(sl.j1, sl.j0 + (int)((16 - reinterpret_cast<uintptr_t>(g + sl.j0) % 16) % 16 / sizeof(T)));
                const int n = (sl.j1 - j0) / VE, j1 = j0 + n * VE;
                if (tid < j0 - sl.j0) g[sl.j0 + tid] = from_f32<T>(0.0f);
                if (tid < sl.j1 - j1) g[j1 + tid] = from_f32<T>(0.0f);
                for (int v = tid; v < n; v += THREADS) reinterpret_cast<uint4*>(g + j0)[v] = make_uint4(0, 0, 0, 0);
            }
        }
    }

    for (; t < a.tokens; buf ^= 1) {
        const int* const slot = slots + buf * K;
        const float* const lq = lqs + buf * K;
        const Slice<T> sl(a, t, rank, log_cluster);
        const int nv = sl.nv;
        const float ahead = weight_ahead(a, t + step, step);
        copies_landed();
        row_ready<THREADS>();
        const float s_t = teacher[buf][0], w = teacher[buf][1];
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
        workers_together<THREADS>();
        const int64_t t_next = live_row(a, t + step, step, ahead);
        const Slice<T> next(a, min(t_next, a.tokens - 1), rank, log_cluster);
        const int nv_next = t_next < a.tokens ? next.nv : 0;
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
            if constexpr (!GRAD) for (int v = tid; v < nv_next; v += THREADS) next.fetch(vec, v, V);
            const float s = warp_sum(sum.x + sum.y);
            if (lane == 0) { part[warp][P_MREST] = m; part[warp][P_SREST] = s; }
        }
        workers_together<THREADS>();
        float2 rest, top;
        float n_top;
        {
            bool in = lane < WARPS;
            rest = join_lanes(in ? part[lane][P_MREST] : -INFINITY, in ? part[lane][P_SREST] : 0.0f, c);
            in = lane < entry_warps;
            top = join_lanes(in ? part[lane][P_MTOP] : -INFINITY, in ? part[lane][P_STOP] : 0.0f, c);
            n_top = warp_sum(in ? part[lane][P_NTOP] : 0.0f);
        }
        if (log_cluster) {
            if (tid < cluster) {
                float* const mine = ranks[rank];
                store_at(mine + P_MREST, tid, rest.x); store_at(mine + P_SREST, tid, rest.y);
                store_at(mine + P_MTOP, tid, top.x); store_at(mine + P_STOP, tid, top.y); store_at(mine + P_NTOP, tid, n_top);
            }
            cluster_barrier();
            const bool in = lane < cluster;
            const float* const r = ranks[in ? lane : 0];
            rest = join_lanes(in ? r[P_MREST] : -INFINITY, in ? r[P_SREST] : 0.0f, c);
            top = join_lanes(in ? r[P_MTOP] : -INFINITY, in ? r[P_STOP] : 0.0f, c);
            n_top = warp_sum(in ? r[P_NTOP] : 0.0f);
        }
        const float m_rest = rest.x, s_rest = rest.y, m = finite_ref(fmaxf(m_rest, top.x));
        const float f_rest = ex2((m_rest - m) * c);                    // 0 when nothing is left out
        const float s = __fmaf_rn(s_rest, f_rest, top.y * ex2((top.x - m) * c));
        const float inv_s = s > 0.0f || s != s ? 1.0f / s : 0.0f;
        const float q_rest = tail && n_top < (float)V ? fmaxf(1.0f - s_t, 0.0f) : 0.0f;
        const float Q = tail ? s_t + q_rest : (s_t > 0.0f || s_t != s_t) ? 1.0f : 0.0f;
        const float scale = w * a.inv_tau;
        if (entries) {      // this slice's share of the loss
            const float log_s = logf(s);
            float l = 0.0f;
            for (int k = tid; k < K; k += estride) {
                if (slot[k] < 0) continue;
                const float q = expf(lq[k]);
                if (q != 0.0f) l += q * (lq[k] - (zk[k] == -INFINITY && s == s ? -INFINITY : (zk[k] - m) * a.inv_tau - log_s));
            }
            l = warp_sum(l);
            if (tid == 0 && rank == 0 && q_rest > 0.0f)
                l += q_rest * (logf(q_rest) - (s_rest > 0.0f ? (m_rest - m) * a.inv_tau + logf(s_rest) - log_s : -INFINITY));
            if (lane == 0) loss_part[warp] = l;
        }
        bool fetched = !GRAD;
        T* const g = GRAD ? static_cast<T*>(a.grad) + t * a.grad_stride : nullptr;
        if constexpr (GRAD) {
            // Left out: p_j (Q - q_rest / p_rest) with p_j = 2^(c (z_j - m_rest)) f_rest / s and p_rest = s_rest f_rest / s.
            const float coef = (Q * f_rest * inv_s - (s_rest > 0.0f ? q_rest / s_rest : 0.0f)) * scale;
            const float2 neg = splat(-finite_ref(m_rest)), c2 = splat(c), coef2 = splat(coef);
            if ((reinterpret_cast<uintptr_t>(g) - reinterpret_cast<uintptr_t>(sl.z)) % 16 == 0) {
                uint4* const dst = reinterpret_cast<uint4*>(g + sl.e0);
                for (int v = tid; v < nv; v += THREADS) {
                    float2 x[VE / 2];
                    to_pairs<T>(vec[v], x);
#pragma unroll
                    for (int i = 0; i < VE / 2; ++i) {
                        const float2 y = mul2_rn(add2_rn(x[i], neg), c2);
                        x[i] = mul2_rn(make_float2(ex2(y.x), ex2(y.y)), coef2);
                    }
                    if (v < nv_next) next.fetch(vec, v, V);
                    if (v >= sl.whole0 && v < sl.whole1) {
                        dst[v] = from_pairs<T>(x);
                    } else {
#pragma unroll
                        for (int i = 0; i < VE; ++i) {
                            const int j = sl.e0 + v * VE + i;
                            if (j >= 0 && j < V) g[j] = from_f32<T>(i & 1 ? x[i / 2].y : x[i / 2].x);
                        }
                    }
                }
                // the next row may have a vector more
                for (int v = tid + (nv - tid + THREADS - 1) / THREADS * THREADS; v < nv_next; v += THREADS) next.fetch(vec, v, V);
                fetched = true;
            } else {
                // The gradient's rows are aligned otherwise than the logits': its own vectors, gathered element by element.
                const int goff = (int)(reinterpret_cast<uintptr_t>(g) % 16 / sizeof(T));
                const int u1 = (sl.j1 + goff + VE - 1) / VE;
#pragma unroll 1
                for (int u = (sl.j0 + goff) / VE + tid; u < u1; u += THREADS) {
                    const int j = u * VE - goff;
                    float2 x[VE / 2];
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        const float zi = j + i >= sl.j0 && j + i < sl.j1 ? to_f32(reinterpret_cast<const T*>(elem)[j + i - sl.e0]) : -INFINITY;
                        (i & 1 ? x[i / 2].y : x[i / 2].x) = ex2((zi + neg.x) * c) * coef;
                    }
                    if (j >= sl.j0 && j + VE <= sl.j1) {
                        *reinterpret_cast<uint4*>(g + j) = from_pairs<T>(x);
                    } else {
#pragma unroll
                        for (int i = 0; i < VE; ++i)
                            if (j + i >= sl.j0 && j + i < sl.j1) g[j + i] = from_f32<T>(i & 1 ? x[i / 2].y : x[i / 2].x);
                    }
                }
            }
        }
        workers_together<THREADS>();        // the listed entries' gradients go over the slice's, and the warps' shares of the loss are there
        if (!fetched) for (int v = tid; v < nv_next; v += THREADS) next.fetch(vec, v, V);
        if constexpr (GRAD) {
            if (entries) {
                const float q_scale = Q * inv_s * scale;
                for (int k = tid; k < K; k += estride) {
                    const int e = slot[k];
                    if (e < 0) continue;
                    float q = 0.0f;
                    if (twice) {
                        for (int i = 0; i < K; ++i) if (slot[i] == e) q += expf(lq[i]);
                    } else {
                        q = expf(lq[k]);
                    }
                    g[sl.e0 + e] = from_f32<T>(__fmaf_rn(ex2((zk[k] - m) * c), q_scale, -q * scale));
                }
            }
        }
        if (warp == 0) {
            const float l = warp_sum(lane < entry_warps ? loss_part[lane] : 0.0f);
            if (lane == 0) {
                if (log_cluster) store_at(&ranks[rank][P_COUNT], 0, l);
                else a.loss[t] = w * l;
            }
        }
        if (log_cluster) {
            cluster_barrier();
            if (rank == 0 && tid == 0) {
                float l = 0.0f;
                for (int r = 0; r < cluster; ++r) l += ranks[r][P_COUNT];
                a.loss[t] = w * l;
            }
        }
        t = t_next;
    }
}

template <typename T, int THREADS, bool GRAD>
cudaError_t launch(const DistillArgs& a, int log_cluster, int slice_vecs, size_t bytes, cudaStream_t s) {
    const int cluster = 1 << log_cluster;
    auto kernel = distill_kernel<T, THREADS, GRAD>;
    cudaError_t e = bytes > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : cudaSuccess;
    if (e != cudaSuccess) return e;
    // As many CTAs as the SMs hold (their registers: see the launch bounds), each on every so manieth row.
    const int per_sm = std::max(1, std::min(blocks_per_sm(THREADS), (int)(227 * 1024 / (bytes + 2048))));
    const int64_t rows = std::min<int64_t>(a.tokens, (148 * per_sm) >> log_cluster);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * cluster));
    cfg.blockDim = dim3(THREADS + 32);
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
    const size_t bytes = (size_t)slice * 16 + (size_t)a.top * 20;
    return with_dtype(logits_dtype, [&](auto t) {
        using T = decltype(t);
        if (slice <= 1024) return a.grad ? launch<T, 128, true>(a, log_cluster, slice, bytes, s) : launch<T, 128, false>(a, log_cluster, slice, bytes, s);
        return a.grad ? launch<T, 256, true>(a, log_cluster, slice, bytes, s) : launch<T, 256, false>(a, log_cluster, slice, bytes, s);
    });
}

}  // namespace lpmm
