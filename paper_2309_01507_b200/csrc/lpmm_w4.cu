// 4-bit weights with group scales: quantizer, dequantizer and the product with a few rows of activations, for sm_100a.
//
// A matrix of `rows` x `cols` keeps its codes row by row, column 2k in bits 0-3 of byte k and column 2k + 1 in bits 4-7 (the
// packing of the optimizer states), rows `codes_stride` bytes apart (a multiple of 16), and one scale and optionally one zero
// point per `group` consecutive columns of a row. Value = (code - zero) * scale, zero = 8 without zero points.
#include <algorithm>
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
//
// y[m, i] = sum over the groups of s (sum over the group's columns of (q - z) x[m, k]): q - z is a small whole number, exact in
// the 16-bit types, so the inner sums run on the tensor cores (m16n8k16, rows of the weight by tokens, binary32 sums) and a
// scale is applied once per group to their result. fp32 activations enter as three bfloat16 parts that add up to them exactly
// (8 significant bits each), as three columns instead of one.
//
// A warp owns 16 rows and streams its codes through a ring of its own in shared memory (cp.async, 256 columns = 2 KB per stage),
// so nothing in the loop waits for another warp. A lane reads one 32-bit word = 8 codes of one row per 32 columns; the pairs
// that its halves hold, (0, 4), (1, 5), (2, 6), (3, 7), are brought to the tensor cores' operand by a mask, an OR with the
// exponent of a power of two and one exact subtraction. The order of the columns inside a product is free as long as both
// operands have the same: the activations are put into shared memory with their pairs in that order.
//
// The columns of a row tile are split over the CTAs of a cluster when there are fewer tiles than the SMs can hold; the ranks'
// sums are added in rank order through distributed shared memory, so results are the same bits every time.

constexpr int kStageCols = 256, kStageBytes = kStageCols / 2;   // columns of one ring stage; its bytes per row
constexpr int kStages = 4;
constexpr int kWarpRing = kStages * 16 * kStageBytes;           // 8 KB
constexpr int kXPad = 64;                                       // bytes between columns: neighbouring columns on other banks

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t r;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ float ld_rank(uint32_t a, uint32_t rank) {    // the same place in CTA `rank`'s shared memory
    float v;
    asm volatile("{\n.reg .b32 t;\nmapa.shared::cluster.u32 t, %1, %2;\nld.shared::cluster.f32 %0, [t];\n}" : "=f"(v) : "r"(a), "r"(rank));
    return v;
}

// Eight codes as four operand registers: (q0, q4), (q1, q5), (q2, q6), (q3, q7), minus the zero point. `zero` and `zero16` come
// from zero_operand().
template <typename M> struct Codes;
template <> struct Codes<__half> {
    // 0x6400 is 1024: OR-ing a code into its low bits adds it, into bits 4-7 adds 16 times it.
    __device__ __forceinline__ static void zero_operand(float z, uint32_t& zero, uint32_t& zero16) {
        zero = pack_pair<__half>(1024.0f + z, 1024.0f + z);
        zero16 = pack_pair<__half>(-64.0f - z, -64.0f - z);
    }
    __device__ __forceinline__ static void expand(uint32_t w, uint32_t zero, uint32_t zero16, uint32_t (&o)[4]) {
        const uint32_t w8 = w >> 8, sixteenth = 0x2c002c00u;
        uint32_t t[4];
        asm("lop3.b32 %0, %1, 0x000f000f, 0x64006400, 0xEA;" : "=r"(t[0]) : "r"(w));
        asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xEA;" : "=r"(t[1]) : "r"(w));
        asm("lop3.b32 %0, %1, 0x000f000f, 0x64006400, 0xEA;" : "=r"(t[2]) : "r"(w8));
        asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xEA;" : "=r"(t[3]) : "r"(w8));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(o[0]) : "r"(t[0]), "r"(zero));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(o[1]) : "r"(t[1]), "r"(sixteenth), "r"(zero16));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(o[2]) : "r"(t[2]), "r"(zero));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(o[3]) : "r"(t[3]), "r"(sixteenth), "r"(zero16));
    }
    __device__ __forceinline__ static void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct Codes<__nv_bfloat16> {
    // 0x4300 is 128 with seven bits of mantissa: only a code in the low four bits fits.
    __device__ __forceinline__ static void zero_operand(float z, uint32_t& zero, uint32_t& zero16) {
        zero = pack_pair<__nv_bfloat16>(128.0f + z, 128.0f + z);
        zero16 = 0;
    }
    __device__ __forceinline__ static void expand(uint32_t w, uint32_t zero, uint32_t, uint32_t (&o)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t t;
            asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xEA;" : "=r"(t) : "r"(w >> (4 * i)));
            asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(o[i]) : "r"(t), "r"(zero));
        }
    }
    __device__ __forceinline__ static void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

template <typename T> struct Operand { using M = T; static constexpr int parts = 1; };
template <> struct Operand<float> { using M = __nv_bfloat16; static constexpr int parts = 3; };

struct W4Product {
    W4Quant w;           // w.w: the activations, w.w_stride: their rows' distance
    int64_t tokens;
    const float* bias;
    void* y;
    int64_t y_stride;
    int32_t scale_dtype, y_f32;
    int32_t block_tokens;   // tokens of one pass over the codes (blockIdx.y)
    int32_t x_cols;         // columns of the activations that shared memory holds at a time (a multiple of 256)
    int32_t x_pitch;        // bytes between its columns (tokens, or parts of them)
};

// GB: 32-column blocks per scale (1, 2 or 4; wider groups repeat their scale). NT: tiles of 8 columns of activations.
template <typename T, int NT, int GB>
__global__ void __launch_bounds__(256) w4_product_kernel(const W4Product p) {
    using M = typename Operand<T>::M;
    constexpr int PARTS = Operand<T>::parts;
    constexpr int NS = GB == 1 ? 2 : 1;         // scales per row, stage and lane
    extern __shared__ __align__(128) unsigned char smem[];
    const W4Quant& a = p.w;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    uint32_t rank, ranks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const int tile_rows = warps * 16;
    const int64_t row0 = (int64_t)(blockIdx.x / ranks) * tile_rows, wrow0 = row0 + warp * 16;
    const int64_t m0 = (int64_t)blockIdx.y * p.block_tokens;
    const int mcount = (int)min((int64_t)p.block_tokens, p.tokens - m0), ncols = mcount * PARTS;
    const int cols = (int)a.cols, all_stages = (cols + kStageCols - 1) / kStageCols;
    const int st0 = (int)((int64_t)all_stages * rank / ranks), st1 = (int)((int64_t)all_stages * (rank + 1) / ranks);
    const int chunk_stages = p.x_cols / kStageCols;

    const uint32_t ring = smem_u32(smem) + warp * kWarpRing;
    const uint32_t xs = smem_u32(smem) + warps * kWarpRing;
    const uint32_t zero_line = xs + (p.block_tokens * PARTS) * p.x_pitch;    // 64 bytes of zeros, read in place of columns that are not there
    if (threadIdx.x < 16) asm volatile("st.shared.u32 [%0], %1;" ::"r"(zero_line + threadIdx.x * 4), "r"(0));

    // Codes: lane l copies 16 bytes of rows l / 8, l / 8 + 4, ...; a row's eight 16-byte pieces are permuted by the row number, so
    // that the eight rows a warp reads at a time lie on different banks.
    const int row_bytes = (cols + 1) / 2;
    const auto fetch = [&](int st) {
        if (st < st1) {
            const uint32_t dst = ring + (st & (kStages - 1)) * (16 * kStageBytes);
            const int byte = st * kStageBytes + (lane & 7) * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 4 + (lane >> 3);
                const bool in = wrow0 + r < a.rows && byte < row_bytes;
                const uint8_t* src = a.codes + (in ? (wrow0 + r) * a.codes_stride + byte : 0);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + r * kStageBytes + (((lane & 7) ^ (r & 7)) << 4)), "l"(src), "r"(in ? 16 : 0) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(st0 + i);

    // Scales (and zero points) of a stage, one stage ahead, in registers: lane t of a row holds groups 2t and 2t + 1 (groups of
    // 32 columns), t (64) or t & 1 (128 and wider) of the stage.
    const int64_t ra = min(wrow0 + g, a.rows - 1) * a.groups, rb = min(wrow0 + g + 8, a.rows - 1) * a.groups;
    const int wide = a.group / 128;
    float sa[NS], sb[NS], za[NS], zb[NS];
    const auto load_scales = [&](int st, float (&sa)[NS], float (&sb)[NS], float (&za)[NS], float (&zb)[NS]) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            int gi = GB == 1 ? st * 8 + 2 * t + i : GB == 2 ? st * 4 + t : (st * 2 + (t & 1)) / wide;
            const bool in = gi < a.groups && st < st1;
            gi = in ? gi : 0;
            sa[i] = in ? load_f32(a.scales, p.scale_dtype, ra + gi) : 0.0f;
            sb[i] = in ? load_f32(a.scales, p.scale_dtype, rb + gi) : 0.0f;
            za[i] = a.zeros ? (float)a.zeros[ra + gi] : 8.0f;
            zb[i] = a.zeros ? (float)a.zeros[rb + gi] : 8.0f;
        }
    };
    load_scales(st0, sa, sb, za, zb);

    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;

    for (int c0 = st0; c0 < st1; c0 += chunk_stages) {
        const int c1 = min(c0 + chunk_stages, st1);
        // Activations of the columns [c0, c1) * 256, eight at a time, in the order of the codes' pairs.
        if (c0 != st0) __syncthreads();
        const int eights = (c1 - c0) * (kStageCols / 8);
        for (int i = threadIdx.x; i < eights * mcount; i += blockDim.x) {
            const int m = i / eights, e = i - m * eights, k = c0 * kStageCols + e * 8;
            const T* row = static_cast<const T*>(a.w) + (m0 + m) * a.w_stride;
            float v[8];
            if (k < cols) load8(row, k, cols, a.vec, v);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = 0.0f;
            }
            uint32_t addr = xs + (m * PARTS) * p.x_pitch + e * 16;
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                uint32_t o[4];
                if constexpr (PARTS == 1) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = pack_pair<M>(v[j], v[j + 4]);
                } else {
                    uint32_t hi[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {      // the upper half of the bits is a bfloat16; what is left is exact
                        hi[j] = __float_as_uint(v[j]) & 0xffff0000u;
                        v[j] = fabsf(v[j]) == INFINITY ? 0.0f : v[j] - __uint_as_float(hi[j]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = (hi[j] >> 16) | hi[j + 4];
                }
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                addr += p.x_pitch;
            }
        }
        __syncthreads();

        uint32_t xaddr[NT], xstep[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool in = n * 8 + g < ncols;
            xaddr[n] = (in ? xs + (n * 8 + g) * p.x_pitch : zero_line) + t * 16;
            xstep[n] = in ? 64 : 0;
        }
        for (int st = c0; st < c1; ++st) {
            fetch(st + kStages - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            __syncwarp();
            float nsa[NS], nsb[NS], nza[NS], nzb[NS];
            load_scales(st + 1, nsa, nsb, nza, nzb);
            const uint32_t codes = ring + (st & (kStages - 1)) * (16 * kStageBytes) + g * kStageBytes + t * 4;
            float part[NT][4];
            float s0 = 0.0f, s1 = 0.0f;
            uint32_t z0 = 0, z0x = 0, z1 = 0, z1x = 0;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                if (b % GB == 0) {        // a new group
                    const int src = (lane & ~3) | (GB == 1 ? b >> 1 : b / GB);
                    const int i = GB == 1 ? b & 1 : 0;
                    s0 = __shfl_sync(0xffffffffu, sa[i], src);
                    s1 = __shfl_sync(0xffffffffu, sb[i], src);
                    if (a.zeros || b == 0) {
                        Codes<M>::zero_operand(a.zeros ? __shfl_sync(0xffffffffu, za[i], src) : 8.0f, z0, z0x);
                        Codes<M>::zero_operand(a.zeros ? __shfl_sync(0xffffffffu, zb[i], src) : 8.0f, z1, z1x);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) part[n][0] = part[n][1] = part[n][2] = part[n][3] = 0.0f;
                }
                uint32_t qa[4], qb[4];
                Codes<M>::expand(lds32(codes + ((b ^ g) << 4)), z0, z0x, qa);
                Codes<M>::expand(lds32(codes + 8 * kStageBytes + ((b ^ g) << 4)), z1, z1x, qb);
                const uint32_t a0[4] = {qa[0], qb[0], qa[1], qb[1]}, a1[4] = {qa[2], qb[2], qa[3], qb[3]};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 x = lds128(xaddr[n]);
                    xaddr[n] += xstep[n];
                    Codes<M>::mma(part[n], a0, x.x, x.y);
                    Codes<M>::mma(part[n], a1, x.z, x.w);
                }
                if (b % GB == GB - 1) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        acc[n][0] = __fmaf_rn(s0, part[n][0], acc[n][0]);
                        acc[n][1] = __fmaf_rn(s0, part[n][1], acc[n][1]);
                        acc[n][2] = __fmaf_rn(s1, part[n][2], acc[n][2]);
                        acc[n][3] = __fmaf_rn(s1, part[n][3], acc[n][3]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) { sa[i] = nsa[i]; sb[i] = nsb[i]; za[i] = nza[i]; zb[i] = nzb[i]; }
            __syncwarp();       // the stage may be overwritten
        }
    }

    // Sums of this CTA, [column][row], into the rings' place; then every rank adds its share of the rows over all ranks.
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float* const red = reinterpret_cast<float*>(smem);
    const int rpitch = tile_rows + 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = n * 8 + 2 * t + (i & 1);
            if (col < ncols) red[col * rpitch + warp * 16 + g + (i >> 1) * 8] = acc[n][i];
        }
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
    else __syncthreads();
    const int share = tile_rows / (int)ranks, r_lo = (int)rank * share;
    for (int i = threadIdx.x; i < share * mcount; i += blockDim.x) {
        const int m = i / share, r = r_lo + i - m * share;
        if (row0 + r >= a.rows) continue;
        float v = 0.0f;
        for (uint32_t k = 0; k < ranks; ++k)
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                const float* at = red + (m * PARTS + part) * rpitch + r;
                v += ranks > 1 ? ld_rank(smem_u32(at), k) : *at;
            }
        if (p.bias) v += p.bias[row0 + r];
        const int64_t o = (m0 + m) * p.y_stride + row0 + r;
        if (p.y_f32) static_cast<float*>(p.y)[o] = v;
        else static_cast<T*>(p.y)[o] = from_f32<T>(v);
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}

template <typename T, int NT, int GB>
cudaError_t launch_product(W4Product p, cudaStream_t s) {
    constexpr int PARTS = Operand<T>::parts;
    const int warps = 8, tile_rows = warps * 16;
    const int64_t tiles = (p.w.rows + tile_rows - 1) / tile_rows, blocks = (p.tokens + p.block_tokens - 1) / p.block_tokens;
    const int stages = (int)((p.w.cols + kStageCols - 1) / kStageCols);
    int ranks = 1;
    while (ranks < 8 && tiles * blocks * ranks < 148 * 2 && stages >= ranks * 4) ranks *= 2;
    const int range = (stages + ranks - 1) / ranks, columns = p.block_tokens * PARTS;
    const int limit = NT <= 2 ? 40 * 1024 : 64 * 1024;
    int chunk = range;
    while (chunk > 1 && (int64_t)columns * (chunk * kStageCols * 2 + kXPad) > limit) chunk = (chunk + 1) / 2;
    p.x_cols = chunk * kStageCols;
    p.x_pitch = p.x_cols * 2 + kXPad;
    const size_t bytes = std::max((size_t)warps * kWarpRing + (size_t)columns * p.x_pitch + 64, (size_t)columns * (tile_rows + 4) * 4);
    auto kernel = w4_product_kernel<T, NT, GB>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * ranks), (unsigned)blocks);
    cfg.blockDim = dim3(warps * 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = ranks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = ranks > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kernel, p);
    return e != cudaSuccess ? e : cudaGetLastError();
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
    return with_dtype(x_dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int PARTS = Operand<T>::parts;
        W4Product p = {};
        p.w = pack_args(m, x, x_stride, sizeof(T));
        p.tokens = tokens; p.bias = bias; p.y = y; p.y_stride = y_stride;
        p.scale_dtype = m.scale_dtype;
        p.y_f32 = y_dtype == 0;
        const int64_t columns = tokens * PARTS;
        const auto run = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            p.block_tokens = (int)std::min<int64_t>(tokens, NT * 8 / PARTS);
            // grid.y counts blocks of tokens and ends at 65535; the rest is another launch's
            const int64_t most = (int64_t)65535 * p.block_tokens;
            for (int64_t done = 0; done < tokens; done += most) {
                W4Product q = p;
                q.tokens = std::min(most, tokens - done);
                q.w.w = static_cast<const T*>(x) + done * x_stride;
                q.y = static_cast<char*>(y) + done * y_stride * (p.y_f32 ? 4 : (int64_t)sizeof(T));
                const cudaError_t e = m.group == 32 ? launch_product<T, NT, 1>(q, s) : m.group == 64 ? launch_product<T, NT, 2>(q, s) : launch_product<T, NT, 4>(q, s);
                if (e != cudaSuccess) return e;
            }
            return cudaSuccess;
        };
        if (columns <= 8) return run(std::integral_constant<int, 1>{});
        if (columns <= 16) return run(std::integral_constant<int, 2>{});
        if (columns <= 32) return run(std::integral_constant<int, 4>{});
        return run(std::integral_constant<int, 8>{});
    });
}

}  // namespace lpmm
