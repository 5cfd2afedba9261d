// Quantisation to microscaled rows and back, and the pre-norm that adds a branch's output to the
// stream and writes its normalised rows in that form (mx.h has the format).
//
// All three are bound by memory: a thread takes eight neighbouring columns (16 or 32 bytes of the
// source), four lanes make a block of 32, whose largest magnitude is two DPP steps.  24576 x 4096 bf16 to e2m1 57 us
// and back 39 us (4.5 and 6.6 TB/s), 200 x 4096 to e4m3 2.6 us.
#include "common.h"
#include "kernels.h"
#include "mx.h"

namespace sgd {

// n / d for n < 2^31 by a multiplication (round-up reciprocal of Granlund and Montgomery, 1994)
struct FastDiv {
    uint32_t d, m, s;
    explicit FastDiv(uint32_t d_) : d(d_), m(0), s(0) {
        while ((1ull << s) < d) ++s;
        m = (uint32_t)((((1ull << 32) * ((1ull << s) - d)) / d) + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(m, n) + n) >> s; }
};

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
    const bf16x8 a = *(const bf16x8*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = bf2f(a[i]);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = f2bf(x[i]);
    *(bf16x8*)p = a;
}

// --------------------------------------------------------------------------- quantisation

template <int FMT, typename T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(MxQuantArgs a, FastDiv groups) {
    const uint32_t n = (uint32_t)a.rows * (uint32_t)(a.K / 8);
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t at = min(i, n - 1);  // a whole row is whole quads: no quad straddles the end
    const uint32_t r = groups.div(at), g = at - r * groups.d;
    float x[8];
    load8((const T*)a.x + (long)r * a.ldx + g * 8, x);
    mx_store8<FMT>(x, r, g, a.rows, a.K, a.codes, a.scales, i < n);
}

template <int FMT, typename T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(MxQuantArgs a, FastDiv groups) {
    const uint32_t n = (uint32_t)a.rows * (uint32_t)(a.K / 8);
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= n) return;
    const uint32_t r = groups.div(i), g = i - r * groups.d;
    const int s = a.scales[mx_scale_at(a.rows, r, g >> 2)];
    // 2^(s - 127): byte 0 is the subnormal 2^-127
    const float f = s == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(s ? (uint32_t)s << 23 : 0x00400000u);
    float x[8];
    if constexpr (FMT == MX_FP4) {
        const uint32_t c = *(const uint32_t*)(a.codes + (long)r * (a.K / 2) + g * 4);
        const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
        const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
        x[0] = v0[0]; x[1] = v0[1]; x[2] = v1[0]; x[3] = v1[1];
        x[4] = v2[0]; x[5] = v2[1]; x[6] = v3[0]; x[7] = v3[1];
    } else {
        const u32x2 c = *(const u32x2*)(a.codes + (long)r * a.K + g * 8);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
            x[4 * h] = lo[0]; x[4 * h + 1] = lo[1]; x[4 * h + 2] = hi[0]; x[4 * h + 3] = hi[1];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= f;
    store8((T*)a.out + (long)r * a.ldx + g * 8, x);
}

hipError_t launch_mx_quantize(int fmt, int bf, const MxQuantArgs& a, hipStream_t st) {
    const FastDiv g((uint32_t)(a.K / 8));
    const dim3 grid((unsigned)(((long)a.rows * (a.K / 8) + 255) / 256));
    if (fmt == MX_FP4) {
        if (bf) mx_quantize_kernel<MX_FP4, bf16><<<grid, 256, 0, st>>>(a, g);
        else mx_quantize_kernel<MX_FP4, float><<<grid, 256, 0, st>>>(a, g);
    } else {
        if (bf) mx_quantize_kernel<MX_FP8, bf16><<<grid, 256, 0, st>>>(a, g);
        else mx_quantize_kernel<MX_FP8, float><<<grid, 256, 0, st>>>(a, g);
    }
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(int fmt, int bf, const MxQuantArgs& a, hipStream_t st) {
    const FastDiv g((uint32_t)(a.K / 8));
    const dim3 grid((unsigned)(((long)a.rows * (a.K / 8) + 255) / 256));
    if (fmt == MX_FP4) {
        if (bf) mx_dequantize_kernel<MX_FP4, bf16><<<grid, 256, 0, st>>>(a, g);
        else mx_dequantize_kernel<MX_FP4, float><<<grid, 256, 0, st>>>(a, g);
    } else {
        if (bf) mx_dequantize_kernel<MX_FP8, bf16><<<grid, 256, 0, st>>>(a, g);
        else mx_dequantize_kernel<MX_FP8, float><<<grid, 256, 0, st>>>(a, g);
    }
    return hipGetLastError();
}

// --------------------------------------------------------------------------- pre-norm
//
// h = x + r (held in x's type), y = h / sqrt(mean(h^2) + eps) w.  The sum of squares, its root and y are in
// fp64: y is rounded once, to 8 or 4 bits, and at fp32 one value in 10^5 or so would fall on the other
// side of a rounding border (or its block's maximum on the other side of a power of two).  The kernel
// waits for memory either way: per value two conversions, one fma and two products in fp64 (8192 x 4096, fp32 stream,
// bf16 branch: 72 us, 5.2 TB/s).

// y as fp32 rounded to odd (the last bit set where anything was cut off): a second rounding to at most
// four bits then gives what one rounding of y would.  Past fp32's range: infinite or NaN, a block of scale 255
__device__ __forceinline__ float round_odd(double y) {
    const uint64_t b = __builtin_bit_cast(uint64_t, y);
    const float f = (float)__builtin_bit_cast(double, b & ~(uint64_t)0x1FFFFFFF);
    return (uint32_t)b & 0x1FFFFFFFu ? __uint_as_float(__float_as_uint(f) | 1u) : f;
}
// The same for values of any size: below 2^-126 fp32 has fewer bits than the mask above leaves, and the conversion rounds
__device__ __forceinline__ float round_odd_small(double y) {
    const float f = (float)fabs(y);
    uint32_t u = __float_as_uint(f);
    if ((double)f > fabs(y)) --u;
    if ((double)__uint_as_float(u) != fabs(y)) u |= 1u;
    return copysignf(__uint_as_float(u), (float)y);
}

// A row's TPR threads hold its 8-column groups g = t + TPR c, c < CH.
template <int FMT, typename TX, typename TR, int TPR, int CH>
__global__ __launch_bounds__(256) void norm_add_mx_kernel(NormMxArgs a) {
    constexpr int RPB = 256 / TPR;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    const long r = (long)blockIdx.x * RPB + rl;
    const bool live = r < a.M;
    const long rr = live ? r : a.M - 1;
    const int ng = a.d / 8;
    float h[CH][8];
    double q = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int g = t + TPR * c;
        if (g < ng) load8((const TX*)a.x + rr * a.d + g * 8, h[c]);
    }
    if (a.r) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int g = t + TPR * c;
            if (g >= ng) continue;
            float u[8];
            load8((const TR*)a.r + rr * a.d + g * 8, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[c][i] += u[i];
                if constexpr (sizeof(TX) == 2) h[c][i] = bf2f(f2bf(h[c][i]));  // the stream is held in its type
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (t + TPR * c >= ng) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) q = fma((double)h[c][i], (double)h[c][i], q);
    }
    q = warp_sum(q);
    if constexpr (TPR > 64) {
        __shared__ double part[4];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = q;
        __syncthreads();
        q = (part[0] + part[1]) + (part[2] + part[3]);
    }
    const double rs = 1.0 / sqrt(q / a.d + (double)a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int g = t + TPR * c;
        const bool in = g < ng;  // the same for the four lanes of a block
        float y[8];
        if (in) {
            float w[8];
            load8(a.w + g * 8, w);
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = round_odd((double)h[c][i] * rs * (double)w[i]);
                top = fmaxf(top, fabsf(y[i]));
            }
            // Beside a value of 2^-107 or more, the first middle between two codes is 2^-125 (e4m3: 2^-18 of its binade): what
            // fp32 rounds, below 2^-126, has code 0 either way
            if (top < 0x1p-107f && top > 0.f)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = round_odd_small((double)h[c][i] * rs * (double)w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = 0.f;
        }
        mx_store8<FMT>(y, rr, in ? g : 0, a.M, a.d, a.codes, a.scales, in && live);
        if (in && live && a.r) store8((TX*)a.xo + rr * a.d + g * 8, h[c]);
    }
}

// A wave a row up to 512 columns, a workgroup a row past that (8192 rows, fp32 + bf16 to e4m3: 256 columns 8.0 us a wave
// and 11.8 a workgroup, 512 columns 10.6 and 12.8, 1024 17.4 and 17.8, 2048 38.0 and 34.0; 64 rows of 2048 5.4 and 3.3)
template <int FMT, typename TX, typename TR>
static void norm_add_types(const NormMxArgs& a, hipStream_t st) {
    if (a.d <= 512) norm_add_mx_kernel<FMT, TX, TR, 64, 1><<<(a.M + 3) / 4, 256, 0, st>>>(a);
    else if (a.d <= 2048) norm_add_mx_kernel<FMT, TX, TR, 256, 1><<<a.M, 256, 0, st>>>(a);
    else if (a.d <= 4096) norm_add_mx_kernel<FMT, TX, TR, 256, 2><<<a.M, 256, 0, st>>>(a);
    else norm_add_mx_kernel<FMT, TX, TR, 256, 4><<<a.M, 256, 0, st>>>(a);
}

template <int FMT>
static void norm_add_fmt(int x_bf, int r_bf, const NormMxArgs& a, hipStream_t st) {
    if (x_bf) r_bf ? norm_add_types<FMT, bf16, bf16>(a, st) : norm_add_types<FMT, bf16, float>(a, st);
    else r_bf ? norm_add_types<FMT, float, bf16>(a, st) : norm_add_types<FMT, float, float>(a, st);
}

hipError_t launch_norm_add_mx(int fmt, int x_bf, int r_bf, const NormMxArgs& a, hipStream_t st) {
    if (fmt == MX_FP4) norm_add_fmt<MX_FP4>(x_bf, r_bf, a, st);
    else norm_add_fmt<MX_FP8>(x_bf, r_bf, a, st);
    return hipGetLastError();
}

}  // namespace sgd
