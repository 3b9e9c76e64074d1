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

constexpr int kDThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_sum(float x) {
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}
template <bool MAX>
__device__ float block_reduce(float x, float* red) {
    x = MAX ? warp_max(x) : warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    x = red[threadIdx.x & (kDThreads / 32 - 1)];
    for (int d = kDThreads / 64; d; d >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, x, d);
        x = MAX ? fmaxf(x, o) : x + o;
    }
    return x;
}

template <typename T, typename U>
__global__ void __launch_bounds__(kDThreads) distill_kernel(const DistillArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int K = a.top, tid = threadIdx.x;
    const int words = (int)((a.vocab + 31) / 32);
    int* ids = reinterpret_cast<int*>(smem);                 // K ids, -1: no entry
    float* lq = reinterpret_cast<float*>(ids + K);           // log2 of the teacher's probabilities
    float* x = lq + K;                                       // c (z_id - max z)
    uint32_t* first = reinterpret_cast<uint32_t*>(x + K);    // 1: the first entry with its id
    uint32_t* bits = first + K;                              // one bit per vocabulary entry: listed
    __shared__ float red[kDThreads / 32];
    __shared__ int dup;
    const float c = a.inv_tau * kLog2e;
    const bool tail = a.teacher_lse != nullptr;

    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const float w = a.weights ? a.weights[t] : 1.0f;
        T* g = a.grad ? static_cast<T*>(a.grad) + t * a.grad_stride : nullptr;
        if (w == 0.0f) {
            if (tid == 0) a.loss[t] = 0.0f;
            if (g) for (int64_t j = tid; j < a.vocab; j += kDThreads) g[j] = from_f32<T>(0.0f);
            continue;
        }
        const T* z = static_cast<const T*>(a.logits) + t * a.logits_stride;
        __syncthreads();
        for (int i = tid; i < words; i += kDThreads) bits[i] = 0;
        if (tid == 0) dup = 0;
        __syncthreads();
        float tmax = -INFINITY;
        for (int k = tid; k < K; k += kDThreads) {
            const int64_t id = a.ids64 ? static_cast<const int64_t*>(a.ids)[t * K + k] : static_cast<const int32_t*>(a.ids)[t * K + k];
            const float tl = to_f32(static_cast<const U*>(a.top_logits)[t * K + k]);
            const bool ok = id >= 0 && id < a.vocab;
            ids[k] = ok ? (int)id : -1;
            lq[k] = ok ? tl : -INFINITY;
            x[k] = ok ? to_f32(z[id]) : 0.0f;
            if (ok) {
                tmax = fmaxf(tmax, tl);
                const uint32_t bit = 1u << (id & 31);
                const bool seen = atomicOr(&bits[id >> 5], bit) & bit;
                first[k] = !seen;
                if (seen) dup = 1;
            } else {
                first[k] = 0;
            }
        }
        __syncthreads();
        // Two classes: the entries left out (without the teacher's log-sum-exp: all of them), and the listed ones.
        const auto left_out = [&](int64_t j) { return !tail || !((bits[j >> 5] >> (j & 31)) & 1u); };
        float m_rest = -INFINITY, m = -INFINITY;
        for (int64_t j = tid; j < a.vocab; j += kDThreads) if (left_out(j)) m_rest = fmaxf(m_rest, to_f32(z[j]));
        m_rest = block_reduce<true>(m_rest, red);
        if (tail) for (int k = tid; k < K; k += kDThreads) if (ids[k] >= 0) m = fmaxf(m, x[k]);
        m = fmaxf(block_reduce<true>(m, red), m_rest);
        const float f_rest = m_rest == -INFINITY ? 0.0f : ex2((m_rest - m) * c);
        const float l_rest = (m_rest - m) * c;
        if (m_rest == -INFINITY) m_rest = 0.0f;
        if (m == -INFINITY) m = 0.0f;
        tmax = block_reduce<true>(tmax, red);
        if (tmax == -INFINITY) tmax = 0.0f;
        if (dup) {     // every id counts once: for its first entry
            for (int k = tid; k < K; k += kDThreads) {
                uint32_t f = ids[k] >= 0;
                for (int i = 0; i < k; ++i) if (ids[i] == ids[k]) f = 0;
                first[k] = f;
            }
        }
        float s_rest = 0.0f, s_top = 0.0f, s_t = 0.0f, n_top = 0.0f;
        for (int64_t j = tid; j < a.vocab; j += kDThreads)
            if (left_out(j)) s_rest += ex2((to_f32(z[j]) - m_rest) * c);
        for (int k = tid; k < K; k += kDThreads) {
            const float xk = (x[k] - m) * c;
            x[k] = xk;
            if (tail && first[k]) { s_top += ex2(xk); n_top += 1.0f; }
            // -infinity stays: its products with the two parts of 1 / tau could cancel to NaN
            const float tl = lq[k];
            const float l = tl == -INFINITY ? tl
                            : tail ? __fmaf_rn(tl, a.inv_tau, __fmaf_rn(tl, a.inv_tau_lo, -a.teacher_lse[t])) * kLog2e : (tl - tmax) * c;
            lq[k] = l;
            s_t += exp2f(l);
        }
        s_rest = block_reduce<false>(s_rest, red);
        s_top = block_reduce<false>(s_top, red);
        s_t = block_reduce<false>(s_t, red);
        n_top = block_reduce<false>(n_top, red);
        const float s = __fmaf_rn(s_rest, f_rest, s_top), log_s = log2f(s), inv_s = s > 0.0f || s != s ? 1.0f / s : 0.0f;
        const float log_t = tail || !(s_t > 0.0f) ? 0.0f : log2f(s_t);
        const float q_rest = tail && n_top < (float)a.vocab ? fmaxf(1.0f - s_t, 0.0f) : 0.0f;
        const float Q = tail ? s_t + q_rest : (s_t > 0.0f || s_t != s_t) ? 1.0f : 0.0f;
        float l = 0.0f;
        for (int k = tid; k < K; k += kDThreads) {
            lq[k] -= log_t;
            const float q = exp2f(lq[k]);
            if (q != 0.0f) l += q * (lq[k] - (x[k] == -INFINITY && s == s ? -INFINITY : x[k] - log_s));
        }
        l = block_reduce<false>(l, red);
        if (q_rest > 0.0f) l += q_rest * (log2f(q_rest) - (s_rest > 0.0f ? l_rest + log2f(s_rest) - log_s : -INFINITY));
        if (tid == 0) a.loss[t] = w * l * kLn2;
        if (!g) continue;
        const float scale = w * a.inv_tau;
        const float coef = (Q * f_rest * inv_s - (s_rest > 0.0f ? q_rest / s_rest : 0.0f)) * scale;
        for (int64_t j = tid; j < a.vocab; j += kDThreads) g[j] = from_f32<T>(ex2((to_f32(z[j]) - m_rest) * c) * coef);
        __syncthreads();
        for (int k = tid; k < K; k += kDThreads) {
            if (ids[k] < 0) continue;
            float q = exp2f(lq[k]);
            if (dup) {
                q = 0.0f;
                for (int i = 0; i < K; ++i) if (ids[i] == ids[k]) q += exp2f(lq[i]);
            }
            g[ids[k]] = from_f32<T>((ex2(x[k]) * inv_s * Q - q) * scale);
        }
    }
}

size_t distill_smem(int64_t vocab, int top) { return (size_t)top * 16 + (size_t)((vocab + 31) / 32) * 4; }

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, int logits_dtype, int top_dtype, cudaStream_t s) {
    return with_dtype(logits_dtype, [&](auto t) {
        return with_dtype(top_dtype, [&](auto u) {
            auto kernel = distill_kernel<decltype(t), decltype(u)>;
            const size_t bytes = distill_smem(a.vocab, a.top);
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (e != cudaSuccess) return e;
            kernel<<<(int)(a.tokens < 148 * 8 ? a.tokens : 148 * 8), kDThreads, bytes, s>>>(a);
            return cudaGetLastError();
        });
    });
}

}  // namespace lpmm
