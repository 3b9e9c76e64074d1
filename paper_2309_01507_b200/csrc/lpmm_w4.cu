// 4-bit weights with group scales: quantizer, dequantizer and the product with a few rows of activations, for sm_100a.
//
// A matrix of `rows` x `cols` keeps its codes row by row, column 2k in bits 0-3 of byte k and column 2k + 1 in bits 4-7 (the
// packing of the optimizer states), rows `codes_stride` bytes apart (a multiple of 16), and one scale and optionally one zero
// point per `group` consecutive columns of a row. Value = (code - zero) * scale, zero = 8 without zero points.
#include <type_traits>

#include "lpmm_internal.h"
#include "lpmm_ops.cuh"

namespace lpmm {

namespace {

constexpr int kW4Threads = 256;

int w4_grid(int64_t blocks) { return (int)(blocks < 1 ? 1 : blocks > 148 * 16 ? 148 * 16 : blocks); }

// ------------------------------------------------------------------------------------------------ quantizer

// Scale of a group from its extremes (lo <= 0 <= hi), rounded to the type it is stored in; binary16 saturates instead of
// overflowing, so that every value stays finite.
template <typename S>
__device__ __forceinline__ float group_scale(float lo, float hi, bool zeros) {
    float s = zeros ? __fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f) : __fmul_rn(fmaxf(hi, -lo), 1.0f / 7.0f);
    if constexpr (std::is_same<S, __half>::value) s = fminf(s, 65504.0f);
    return to_f32(from_f32<S>(s));
}
__device__ __forceinline__ float group_zero(float lo, float rcp, bool zeros) {
    return zeros ? fminf(fmaxf(rintf(__fmul_rn(-lo, rcp)), 0.0f), 15.0f) : 8.0f;
}
__device__ __forceinline__ uint32_t w4_code(float w, float rcp, float zero) {
    return (uint32_t)fminf(fmaxf(__fadd_rn(rintf(__fmul_rn(w, rcp)), zero), 0.0f), 15.0f);
}

// Eight consecutive elements of a row from column c on; zeros behind the row's end.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, bool vec, float (&v)[8]) {
    if (vec && c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(row + c)), b = __ldg(reinterpret_cast<const float4*>(row + c) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(row + c));
            const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 p = unpack_pair<T>(u[i]);
                v[2 * i] = p.x; v[2 * i + 1] = p.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (c + i < cols) ? to_f32(row[c + i]) : 0.0f;
    }
}

struct W4Quant {
    const void* w;
    int64_t w_stride;
    uint8_t* codes;
    void* scales;
    uint8_t* zeros;
    int64_t rows, cols, codes_stride, groups;
    int32_t group, vec;
};

// One warp per `span` columns of a row, a lane owns eight consecutive columns (one 32-bit word of codes). Groups of 32, 64 and
// 128 columns are 4, 8 and 16 neighbouring lanes; wider groups (multiples of 128) are walked twice by one warp.
template <typename T, typename S>
__global__ void __launch_bounds__(kW4Threads) w4_quantize_kernel(const W4Quant a) {
    const int lane = threadIdx.x & 31;
    const int64_t span = a.group > 128 ? a.group : 256;
    const int64_t chunks = (a.cols + span - 1) / span;
    const int lanes = a.group > 128 ? 32 : a.group / 8;
    const int64_t items = a.rows * chunks;
    for (int64_t it = (int64_t)blockIdx.x * (kW4Threads / 32) + (threadIdx.x >> 5); it < items; it += (int64_t)gridDim.x * (kW4Threads / 32)) {
        const int64_t r = it / chunks, c0 = (it - r * chunks) * span;
        const T* row = static_cast<const T*>(a.w) + r * a.w_stride;
        const int64_t end = min(c0 + span, a.cols);
        float v[8], lo = 0.0f, hi = 0.0f;
        for (int64_t c = c0 + lane * 8; c < end; c += 256) {
            load8(row, c, end, a.vec, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); }
        }
        for (int d = lanes >> 1; d; d >>= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        }
        const float s = group_scale<S>(lo, hi, a.zeros != nullptr);
        const float rcp = scale_rcp(s), zero = group_zero(lo, rcp, a.zeros != nullptr);
        const int64_t c1 = c0 + lane * 8;
        if (c1 < end && (lane & (lanes - 1)) == 0) {
            const int64_t g = r * a.groups + c1 / a.group;
            static_cast<S*>(a.scales)[g] = from_f32<S>(s);
            if (a.zeros) a.zeros[g] = (uint8_t)zero;
        }
        for (int64_t c = c1; c < end; c += 256) {
            if (span > 256) load8(row, c, end, a.vec, v);
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) word |= (c + i < end ? w4_code(v[i], rcp, zero) : 0u) << (4 * i);
            *reinterpret_cast<uint32_t*>(a.codes + r * a.codes_stride + (c >> 1)) = word;
        }
    }
}

// ---------------------------------------------------------------------------------------------- dequantizer

template <typename T, typename S>
__global__ void __launch_bounds__(kW4Threads) w4_dequantize_kernel(const W4Quant a, T* __restrict__ out, int64_t out_stride) {
    const int64_t words = (a.cols + 7) / 8;
    const int64_t items = a.rows * words;
    for (int64_t it = (int64_t)blockIdx.x * kW4Threads + threadIdx.x; it < items; it += (int64_t)gridDim.x * kW4Threads) {
        const int64_t r = it / words, c = (it - r * words) * 8;
        const uint32_t q = __ldg(reinterpret_cast<const uint32_t*>(a.codes + r * a.codes_stride + (c >> 1)));
        const int64_t g = r * a.groups + c / a.group;
        const float s = to_f32(static_cast<const S*>(a.scales)[g]), z = a.zeros ? (float)a.zeros[g] : 8.0f;
        T* o = out + r * out_stride + c;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(__fsub_rn((float)((q >> (4 * i)) & 15u), z), s);
        if (a.vec && c + 8 <= a.cols) {
            if constexpr (sizeof(T) == 4) {
                reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                *reinterpret_cast<uint4*>(o) = make_uint4(pack_pair<T>(v[0], v[1]), pack_pair<T>(v[2], v[3]), pack_pair<T>(v[4], v[5]), pack_pair<T>(v[6], v[7]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (c + i < a.cols) o[i] = from_f32<T>(v[i]);
        }
    }
}

// -------------------------------------------------------------------------------------------------- product

// One warp per output row and group of four tokens, fp32 multiply-adds; a lane owns eight consecutive columns.
template <typename T, typename S, typename Y>
__global__ void __launch_bounds__(kW4Threads) w4_matvec_kernel(const W4Quant a, const T* __restrict__ x, int64_t x_stride, int64_t tokens,
                                                              const float* __restrict__ bias, Y* __restrict__ y, int64_t y_stride) {
    const int lane = threadIdx.x & 31;
    const int64_t blocks = (tokens + 3) / 4, items = a.rows * blocks;
    for (int64_t it = (int64_t)blockIdx.x * (kW4Threads / 32) + (threadIdx.x >> 5); it < items; it += (int64_t)gridDim.x * (kW4Threads / 32)) {
        const int64_t r = it / blocks, m0 = (it - r * blocks) * 4;
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t c = lane * 8; c < a.cols; c += 256) {
            const uint32_t q = __ldg(reinterpret_cast<const uint32_t*>(a.codes + r * a.codes_stride + (c >> 1)));
            const int64_t g = r * a.groups + c / a.group;
            const float s = to_f32(static_cast<const S*>(a.scales)[g]), z = a.zeros ? (float)a.zeros[g] : 8.0f;
            for (int m = 0; m < 4 && m0 + m < tokens; ++m) {
                float v[8], part = 0.0f;
                load8(x + (m0 + m) * x_stride, c, a.cols, false, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) part = __fmaf_rn((float)((q >> (4 * i)) & 15u) - z, v[i], part);
                acc[m] = __fmaf_rn(s, part, acc[m]);
            }
        }
        for (int m = 0; m < 4 && m0 + m < tokens; ++m) {
            float t = acc[m];
            for (int d = 16; d; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
            if (lane == 0) y[(m0 + m) * y_stride + r] = from_f32<Y>(bias ? t + bias[r] : t);
        }
    }
}

W4Quant pack_args(const W4Matrix& m, const void* w, int64_t stride, int es) {
    const bool vec = (reinterpret_cast<uintptr_t>(w) % 16 == 0) && (stride * es % 16 == 0);
    return {w, stride, m.codes, m.scales, m.zeros, m.rows, m.cols, m.codes_stride, (m.cols + m.group - 1) / m.group, m.group, vec};
}

}  // namespace

cudaError_t launch_w4_quantize(const W4Matrix& m, const void* w, int dtype, int64_t w_stride, cudaStream_t s) {
    const int64_t span = m.group > 128 ? m.group : 256;
    const int grid = w4_grid((m.rows * ((m.cols + span - 1) / span) + 7) / 8);
    return with_dtype(dtype, [&](auto t) {
        return with_dtype(m.scale_dtype, [&](auto sc) {
            w4_quantize_kernel<decltype(t), decltype(sc)><<<grid, kW4Threads, 0, s>>>(pack_args(m, w, w_stride, sizeof(t)));
            return cudaGetLastError();
        });
    });
}

cudaError_t launch_w4_dequantize(const W4Matrix& m, void* out, int dtype, int64_t out_stride, cudaStream_t s) {
    const int grid = w4_grid((m.rows * ((m.cols + 7) / 8) + kW4Threads - 1) / kW4Threads);
    return with_dtype(dtype, [&](auto t) {
        return with_dtype(m.scale_dtype, [&](auto sc) {
            using T = decltype(t);
            w4_dequantize_kernel<T, decltype(sc)><<<grid, kW4Threads, 0, s>>>(pack_args(m, out, out_stride, sizeof(T)), static_cast<T*>(out), out_stride);
            return cudaGetLastError();
        });
    });
}

cudaError_t launch_w4_matvec(const W4Matrix& m, const void* x, int x_dtype, int64_t x_stride, int64_t tokens, const float* bias,
                             void* y, int y_dtype, int64_t y_stride, cudaStream_t s) {
    const int grid = w4_grid((m.rows * ((tokens + 3) / 4) + 7) / 8);
    return with_dtype(x_dtype, [&](auto t) {
        return with_dtype(m.scale_dtype, [&](auto sc) {
            using T = decltype(t);
            const W4Quant a = pack_args(m, x, x_stride, sizeof(T));
            if (y_dtype == x_dtype) w4_matvec_kernel<T, decltype(sc), T><<<grid, kW4Threads, 0, s>>>(a, static_cast<const T*>(x), x_stride, tokens, bias, static_cast<T*>(y), y_stride);
            else w4_matvec_kernel<T, decltype(sc), float><<<grid, kW4Threads, 0, s>>>(a, static_cast<const T*>(x), x_stride, tokens, bias, static_cast<float*>(y), y_stride);
            return cudaGetLastError();
        });
    });
}

}  // namespace lpmm
