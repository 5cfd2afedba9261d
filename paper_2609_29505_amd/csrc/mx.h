// Microscaled rows: e4m3 or e2m1 elements with one power-of-two scale per 32 columns (the OCP
// Microscaling formats), as the quantisation, the pre-norm and the product hold them.
//
// Codes are row-major and compact: K bytes a row (e4m3) or K / 2 (e2m1, the even column in the low
// four bits).  Scale bytes (value 2^(byte - 127), 255: NaN) lie in chunks of eight blocks,
// [ceil(K / 256)][rows][8], so that the eight bytes that a row's 256 columns need are one 8-byte word and
// a tile's rows are one contiguous piece: a product's workgroup loads 256 rows' scales of a k tile as
// 2 KB, where a row-major [rows][K / 32] layout would touch one cache line per row.
#pragma once

#include "common.h"

namespace sgd {

// byte of block b (of 32 columns) of row r
__host__ __device__ __forceinline__ long mx_scale_at(long rows, long r, int b) { return ((long)(b >> 3) * rows + r) * 8 + (b & 7); }

template <int FMT> struct MxFmt;
template <> struct MxFmt<MX_FP8> { static constexpr int EMAX = 8; };  // largest value 448 = 1.75 2^8
template <> struct MxFmt<MX_FP4> { static constexpr int EMAX = 2; };  // largest value 6 = 1.5 2^2

// Scale byte of a block whose largest magnitude has the bits `big`: 2^(floor(log2 |x|) - EMAX), not below
// 2^-127; 255 if the block holds a NaN or an infinity (their bits are the largest).
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t big) {
    const int e = (int)(big >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - MxFmt<FMT>::EMAX, 0);
}

// Codes of eight values with scale byte s: x 2^(127 - s) is exact, then one rounding to the format
// (nearest even; values past the largest saturate, which only the top of the block's own binade is).
// Returns one word (e2m1) in c[0], or two (e4m3).
template <int FMT>
__device__ __forceinline__ void mx_encode8(const float (&x)[8], uint32_t s, uint32_t (&c)[2]) {
    const float up = s == 255 ? 0.f : __uint_as_float((254u - s) << 23);  // 2^(127 - s); a NaN block's codes are 0
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = s == 255 ? 0.f : x[i] * up;
    if constexpr (FMT == MX_FP4) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
        c[0] = w;
        c[1] = 0;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i], -448.f, 448.f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
            c[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], w, true);
        }
    }
}

// largest of v over the four lanes of a quad (DPP): a block of 32 columns, eight a lane
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true));
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true));
}

// Quantises the eight values x of 8-column group g of row r (four neighbouring lanes hold a block, and all
// of them call this) and stores them; the lane of the row's last block also clears the bytes that pad
// its chunk.  store: whether this lane's group exists (the same for the four lanes).
template <int FMT>
__device__ __forceinline__ void mx_store8(const float (&x)[8], long r, int g, long rows, int K, uint8_t* codes,
                                          uint8_t* scales, bool store) {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max(big, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    const uint32_t s = mx_scale_byte<FMT>(quad_max(big));
    uint32_t c[2];
    mx_encode8<FMT>(x, s, c);
    if (!store) return;
    if constexpr (FMT == MX_FP4) *(uint32_t*)(codes + r * (K / 2) + g * 4) = c[0];
    else *(u32x2*)(codes + r * K + g * 8) = u32x2{c[0], c[1]};
    if ((g & 3) == 0) {
        const int b = g >> 2;
        uint8_t* const at = scales + mx_scale_at(rows, r, b);
        at[0] = (uint8_t)s;
        if (b + 1 == K / 32)
            for (int i = 1; i < 8 - (b & 7); ++i) at[i] = 0;
    }
}

}  // namespace sgd
