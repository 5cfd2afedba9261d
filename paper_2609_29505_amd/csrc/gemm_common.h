// Pieces that the matrix-core GEMMs share (bf16 and microscaled): the loads straight into LDS and
// their waits, the order of weight rows in a tile, and the epilogues.
#pragma once

#include <type_traits>
#include <utility>

#include "common.h"
#include "kernels.h"

namespace sgd {

// Rotary head projections: the q and k product columns of each head are taken in the order
// (0, dh/2, 1, dh/2 + 1, ...), so the two dims of every rotary pair are adjacent columns and a
// block tile of any even width holds whole pairs.  Column n of the product is weight row (and
// bias entry) rope_row(n); v columns (n >= vstart) keep their order.
__device__ __forceinline__ long rope_row(long n, int dh, long vstart) {
    if (n >= vstart) return n;
    const int hl = (int)(n % dh);
    return n - hl + ((hl & 1) ? dh / 2 + hl / 2 : hl / 2);
}

template <int I> using IntC = std::integral_constant<int, I>;

// f(IntC<0>{}), ..., f(IntC<N - 1>{})
template <class Fn, int... I>
__device__ __forceinline__ void static_for_impl(Fn& f, std::integer_sequence<int, I...>) {
    (f(IntC<I>{}), ...);
}
template <int N, class Fn>
__device__ __forceinline__ void static_for(Fn&& f) {
    static_for_impl(f, std::make_integer_sequence<int, N>{});
}

// --------------------------------------------------------------------------- epilogue
//
// Straight from the accumulators, without LDS or a barrier.  In the MFMA output layout lane l holds
// column l % 32 of a 32 x 32 block and, in registers 4 q .. 4 q + 3, its rows 8 q + 4 (l / 32) +
// 0..3.  Which product column a block column stands for is the loader's choice (it picks the weight
// row for each LDS row), and it is made so that a lane's values of one row are neighbours
// (tile_col): two blocks side by side give a lane columns 2 l and 2 l + 1.  The pairs of a rotary
// head and the gate and up columns of a gated MLP then meet in one lane, four consecutive tokens of
// a V^T row are four registers, and a transpose of the four rows within a quad of lanes (DPP) leaves
// each lane eight neighbouring columns of one row: 16-byte stores that fill whole 128-byte lines.
//
// Every batch of rows loads its global operands (h, delta, gate) before its first store: a loop
// that alternates them waits for each store (vmcnt counts both).
//
// An epilogue's cost beyond its bytes is what a launch with K = 64 shows (8192 rows, 256 x 256
// tiles): staged through LDS in 128-row chunks 28.9 us plain, 42.7 GELU(erf), 21.5 residual (1024
// columns), 56.5 GEGLU; this one 24.1, 34.8, 19.9 and 48.4.

__device__ __forceinline__ void store_bf16x4(bf16* dst, const float v[4]) {
    bf16x4 s;
    s[0] = f2bf(v[0]); s[1] = f2bf(v[1]); s[2] = f2bf(v[2]); s[3] = f2bf(v[3]);
    *(bf16x4*)dst = s;
}

template <int ACT>
__device__ __forceinline__ float act_fn(float x) {
    if (ACT == ACT_GELU_ERF) return gelu_erf(x);
    if (ACT == ACT_GELU_TANH) return gelu_tanh(x);
    if (ACT == ACT_SILU) return silu(x);
    return x;
}

// calls f(tag) with the activation as a compile-time constant
template <class Fn>
__device__ __forceinline__ void with_act(int act, Fn&& f) {
    switch (act) {
        case ACT_GELU_ERF: f(IntC<ACT_GELU_ERF>{}); break;
        case ACT_GELU_TANH: f(IntC<ACT_GELU_TANH>{}); break;
        case ACT_SILU: f(IntC<ACT_SILU>{}); break;
        default: f(IntC<ACT_NONE>{}); break;
    }
}

// Column (of a wave's TN x 32) of lane column l in MFMA block j: blocks are taken in pairs whose
// columns interleave; a last single block keeps its order.
template <int TN>
__device__ __forceinline__ int tile_col(int j, int l) {
    return j < TN / 2 * 2 ? j / 2 * 64 + 2 * l + (j & 1) : j * 32 + l;
}
// Gated products: hidden column (of a wave's TN x 16) of lane column l in block j, and whether it
// is the up half.  Gate block j pairs with up block j + (TN + 1) / 2; the middle block of an odd TN
// holds 16 gate columns and then their 16 up columns.
template <int TN>
__device__ __forceinline__ int gated_col(int j, int l, bool& up) {
    constexpr int H = TN / 2, UP = (TN + 1) / 2;
    if (TN % 2 && j == H) { up = l >= 16; return H * 32 + (l & 15); }
    up = j >= UP;
    return (up ? j - UP : j) * 32 + l;
}

// Weight row of LDS row r of column tile tn (every kernel's B loader)
template <class C>
__device__ __forceinline__ long weight_row(const EpiParams& ep, int F, int tn, int r) {
    const int w = r / C::WN, x = r - w * C::WN, j = x >> 5, l = x & 31;
    if (ep.kind == EP_GATED) {
        bool up;
        const int c = gated_col<C::TN>(j, l, up);
        return (long)tn * (C::BN / 2) + w * (C::WN / 2) + c + (up ? F : 0);
    }
    const long n = (long)tn * C::BN + w * C::WN + tile_col<C::TN>(j, l);
    if (ep.kind == EP_HEADS && ep.rope) return rope_row(n, ep.dh, (long)(2 - ep.which0) * ep.d);
    return n;
}

// 4 x 4 transpose of 32-bit values within each quad of lanes: v[k] of lane q becomes v[q] of lane k
// (DPP quad permutes; every lane of the quad active).
__device__ __forceinline__ uint32_t quad_xor1(uint32_t x) { return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t quad_xor2(uint32_t x) { return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xF, 0xF, true); }
__device__ __forceinline__ void quad_transpose(uint32_t (&v)[4], int l) {
    const bool o1 = l & 1, o2 = l & 2;
    uint32_t a[4];
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const uint32_t x = quad_xor1(v[k + 1]), y = quad_xor1(v[k]);
        a[k] = o1 ? x : v[k];
        a[k + 1] = o1 ? v[k + 1] : y;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t x = quad_xor2(a[k + 2]), y = quad_xor2(a[k]);
        v[k] = o2 ? x : a[k];
        v[k + 2] = o2 ? a[k + 2] : y;
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    bf16x2 s;
    s[0] = f2bf(x);
    s[1] = f2bf(y);
    return __builtin_bit_cast(uint32_t, s);
}

// two bf16 values at p (4-byte aligned)
__device__ __forceinline__ void put2(bf16* p, const float* v) { *(uint32_t*)p = pack_bf16(v[0], v[1]); }

template <class C>
__device__ __forceinline__ void epilogue(f32x16 (&acc)[C::TM][C::TN], const GemmArgs& g, const EpiParams& ep, int m0,
                                         int tn, int wm, int wn, int split) {
    constexpr int TM = C::TM, TN = C::TN;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // nothing derived from it is computed before the main loop
    const int l = tid & 31, lhalf = (tid >> 5) & 1, lq = l & 3;
    // first of the four rows of registers 4 q .. 4 q + 3 of MFMA block i
    auto row_of = [&](int i, int q) { return m0 + C::block_row(wm, i) + lhalf * 4 + q * 8; };
    // sample of a row: floor((row + 0.5) / ntok) in fp32 is exact while row < 2^21
    const float rntok = 1.0f / (float)ep.ntok;
    auto sample_of = [&](int row) { return (int)(((float)row + 0.5f) * rntok); };
    // bf16 values o[u] of rows row0 + u, u < 4, column c of this lane -> after a quad transpose the
    // lane holds row row0 + l % 4 and four columns of its quad, from c - l % 4 on (dst: that place)
    auto quad_single = [&](const float (&o)[4]) {
        uint32_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = __float_as_uint(o[u]);
        quad_transpose(v, l);
        return u32x2{pack_bf16(__uint_as_float(v[0]), __uint_as_float(v[1])),
                     pack_bf16(__uint_as_float(v[2]), __uint_as_float(v[3]))};
    };

    if (ep.kind == EP_GATED) {
        const int F = ep.F, c0 = tn * (C::BN / 2) + wn * (C::WN / 2);
        float b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            bool up;
            const int c = gated_col<TN>(j, l, up);
            b[j] = ep.bias ? ep.bias[c0 + c + (up ? F : 0)] : 0.f;
        }
        with_act(ep.act, [&](auto actc) {
            constexpr int ACT = decltype(actc)::value;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = row_of(i, q) + lq;
                    bf16* const out = (bf16*)ep.out + (long)row * ep.ldo + c0 + (l & ~3);
                    constexpr int H = TN / 2;
                    // gate block j pairs with up block j + (TN + 1) / 2
#pragma unroll
                    for (int j = 0; j < H; ++j) {
                        constexpr int UP = (TN + 1) / 2;
                        float o[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            o[u] = act_fn<ACT>(acc[i][j][q * 4 + u] + b[j]) * (acc[i][UP + j][q * 4 + u] + b[UP + j]);
                        const u32x2 s = quad_single(o);
                        if (row < g.M) *(u32x2*)(out + j * 32) = s;
                    }
                    if constexpr (TN % 2) {
                        // lanes 0..15 of the middle block hold gate columns, 16..31 their up columns
                        float o[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const float x = acc[i][H][q * 4 + u] + b[H];
                            const float y = __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F));  // l ^ 16
                            o[u] = act_fn<ACT>(x) * y;
                        }
                        const u32x2 s = quad_single(o);
                        if (l < 16 && row < g.M) *(u32x2*)(out + H * 32) = s;
                    }
                }
        });
        return;
    }

    // column groups: a pair of neighbouring columns from blocks j, j + 1 (V = 2), or one column of a
    // last single block (V = 1)
    const int nw = tn * C::BN + wn * C::WN;  // the wave's first product column
    auto groups = [&](auto&& f) {
        if constexpr (TN >= 2) f(IntC<0>{}, IntC<2>{}, nw + 2 * l);
        if constexpr (TN >= 4) f(IntC<2>{}, IntC<2>{}, nw + 64 + 2 * l);
        if constexpr (TN % 2) f(IntC<TN - 1>{}, IntC<1>{}, nw + (TN - 1) * 32 + l);
    };
    // rows row0 .. row0 + 3 of a group's columns n .. n + V - 1 as bf16: one store of the quad's 4 V
    // columns of row row0 + l % 4 at dst (a pointer to column n - V (l % 4) of that row); cols: how
    // many of them exist (a multiple of 4; <= 0: none)
    auto store_quad = [&](auto vc, bf16* dst, const float (*o)[decltype(vc)::value], int cols) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V == 2) {
            uint32_t v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = pack_bf16(o[u][0], o[u][1]);
            quad_transpose(v, l);
            if (cols >= 8) *(u32x4*)dst = u32x4{v[0], v[1], v[2], v[3]};
            else if (cols >= 4) *(u32x2*)dst = u32x2{v[0], v[1]};
        } else {
            const float t[4] = {o[0][0], o[1][0], o[2][0], o[3][0]};
            const u32x2 s = quad_single(t);
            if (cols >= 4) *(u32x2*)dst = s;
        }
    };

    if (ep.kind == EP_ACT) {
        groups([&](auto jc, auto vc, int n) {
            constexpr int J = decltype(jc)::value, V = decltype(vc)::value;
            float b[V];
#pragma unroll
            for (int v = 0; v < V; ++v) b[v] = ep.bias && n < g.N ? ep.bias[n + v] : 0.f;
            const int nq = n - V * lq;
            with_act(ep.act, [&](auto actc) {
                constexpr int ACT = decltype(actc)::value;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    float rb[V] = {};
                    int bs = -1;  // sample whose row bias rb holds (rows rise: it changes rarely)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int row0 = row_of(i, q);
                        float o[4][V];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            if (ACT == ACT_NONE && ep.rowbias) {
                                const int s = sample_of(min(row0 + u, g.M - 1));
                                if (s != bs && n < g.N)
#pragma unroll
                                    for (int v = 0; v < V; ++v) rb[v] = ep.rowbias[(long)s * ep.rowbias_ld + n + v];
                                bs = s;
                            }
#pragma unroll
                            for (int v = 0; v < V; ++v) o[u][v] = act_fn<ACT>((acc[i][J + v][q * 4 + u] + b[v]) + rb[v]);
                        }
                        const int row = row0 + lq;
                        store_quad(vc, (bf16*)ep.out + (long)row * ep.ldo + nq, o, row < g.M ? g.N - nq : 0);
                    }
                }
            });
        });
    } else if (ep.kind == EP_HEADS) {
        const int vstart = (2 - ep.which0) * ep.d;  // first v^T product column
        bf16* const qptr = (bf16*)ep.q;
        bf16* const kptr = (bf16*)ep.k;
        bf16* const vt = (bf16*)ep.vt;
        groups([&](auto jc, auto vc, int n) {
            constexpr int J = decltype(jc)::value, V = decltype(vc)::value;
            if (n >= g.N) return;
            if (n >= vstart) {
                // V^T: four consecutive tokens of a row per store
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int nv = n + v - vstart, vh = nv / ep.dh, vj = nv - vh * ep.dh;
                    const float bv = ep.bias ? ep.bias[n + v] : 0.f;
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int row0 = row_of(i, q);
                            if (row0 >= g.M) continue;
                            const int bs0 = sample_of(row0), tok0 = row0 - bs0 * ep.ntok;
                            float o[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u) o[u] = acc[i][J + v][q * 4 + u] + bv;
                            if (tok0 % 4 == 0 && tok0 + 3 < ep.ntok && row0 + 3 < g.M) {
                                store_bf16x4(vt + (((long)bs0 * ep.H + vh) * ep.dh + vj) * ep.np + tok0, o);
                            } else {
                                // two tokens at a time where they stay together (an even sample length)
#pragma unroll
                                for (int u = 0; u < 4; u += 2) {
                                    const int row = row0 + u;
                                    if (row >= g.M) break;
                                    const int bs = sample_of(row), tok = row - bs * ep.ntok;
                                    bf16* const dst = vt + (((long)bs * ep.H + vh) * ep.dh + vj) * ep.np + tok;
                                    if (tok % 2 == 0 && tok + 1 < ep.ntok && row + 1 < g.M) {
                                        put2(dst, o + u);
                                        continue;
                                    }
                                    dst[0] = f2bf(o[u]);
                                    if (row + 1 >= g.M) break;
                                    const int bs1 = sample_of(row + 1), tok1 = row + 1 - bs1 * ep.ntok;
                                    vt[(((long)bs1 * ep.H + vh) * ep.dh + vj) * ep.np + tok1] = f2bf(o[u + 1]);
                                }
                            }
                        }
                }
                return;
            }
            // q / k columns.  Quads of lanes share one head: d, vstart and dh are multiples of 8 (or
            // dh of 4 only, whose columns are stored one by one below)
            const int proj = ep.which0 + n / ep.d, nn = n - (proj - ep.which0) * ep.d;
            const int hh = nn / ep.dh, j = nn - hh * ep.dh;
            bf16* const base = (proj == 0 ? qptr : kptr) + (long)hh * ep.np * ep.dh;
            const long bstride = (long)ep.H * ep.np * ep.dh;
            if (!ep.rope) {
                float b[V];
#pragma unroll
                for (int v = 0; v < V; ++v) b[v] = ep.bias ? ep.bias[n + v] : 0.f;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int row0 = row_of(i, q);
                        float o[4][V];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int v = 0; v < V; ++v) o[u][v] = acc[i][J + v][q * 4 + u] + b[v];
                        if (ep.dh % 8 == 0) {
                            const int row = row0 + lq, bs = sample_of(row), tok = row - bs * ep.ntok;
                            store_quad(vc, base + bs * bstride + (long)tok * ep.dh + j - V * lq, o, row < g.M ? 8 : 0);
                        } else {
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const int row = row0 + u, bs = sample_of(row), tok = row - bs * ep.ntok;
                                if (row >= g.M) break;
#pragma unroll
                                for (int v = 0; v < V; ++v) base[bs * bstride + (long)tok * ep.dh + j + v] = f2bf(o[u][v]);
                            }
                        }
                    }
                return;
            }
            // rotary columns (pairs adjacent, see rope_row): product columns 2 p and 2 p + 1 of a
            // head hold dims p and p + dh/2.  A group of two is a whole pair; in a single block the
            // pair's other column is in lane l ^ 1.  The angle is the fractional turn of token x
            // inverse frequency (v_sin_f32 / v_cos_f32 take turns); the turn count carries ~1e-4 rad
            // of fp32 rounding at 1024 tokens, far below the bf16 resolution of the output
            const int hd = ep.dh / 2, pj = j / 2;
            float b[V];
#pragma unroll
            for (int v = 0; v < V; ++v) b[v] = ep.bias ? ep.bias[rope_row(n + v, ep.dh, vstart)] : 0.f;
            const float invt = exp2f(-(2.0f * (float)pj / (float)ep.dh) * ep.rope_log2_theta) * 0.159154943091895336f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row0 = row_of(i, q);
                    float o1[4], o2[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int bs = sample_of(row0 + u), tok = row0 + u - bs * ep.ntok;
                        const float t = (float)tok * invt;
                        const float f = t - rintf(t);
                        const float sn = __builtin_amdgcn_sinf(f), cs = __builtin_amdgcn_cosf(f);
                        const float x = acc[i][J][q * 4 + u] + b[0];
                        if constexpr (V == 2) {
                            const float x2 = acc[i][J + 1][q * 4 + u] + b[1];
                            o1[u] = x * cs - x2 * sn;
                            o2[u] = x2 * cs + x * sn;
                        } else {
                            const float y = __uint_as_float(quad_xor1(__float_as_uint(x)));
                            o1[u] = (l & 1) ? x * cs + y * sn : x * cs - y * sn;
                        }
                    }
                    if constexpr (V == 2) {
                        // four neighbouring pairs of token row0 + l % 4: dims p .. p + 3 and their partners
                        const u32x2 s1 = quad_single(o1), s2 = quad_single(o2);
                        const int row = row0 + lq, bs = sample_of(row), tok = row - bs * ep.ntok;
                        bf16* const dst = base + bs * bstride + (long)tok * ep.dh + pj - lq;
                        if (row < g.M) {
                            *(u32x2*)dst = s1;
                            *(u32x2*)(dst + hd) = s2;
                        }
                    } else {
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int row = row0 + u, bs = sample_of(row), tok = row - bs * ep.ntok;
                            if (row < g.M) base[bs * bstride + (long)tok * ep.dh + pj + ((l & 1) ? hd : 0)] = f2bf(o1[u]);
                        }
                    }
                }
        });
    } else {
        // EP_RESID: v = (acc + bias) [* gate]; h = hin + v; delta = v | delta += v; hcopy = bf16(h);
        //           the last of a step: z <- alpha z - beta h in place of h's store
        // EP_SKIP:  h = acc + bias [+ cached delta]; hcopy = bf16(h)
        // EP_PARTIAL: part s = acc (+ bias in range 0), as EP_SKIP into h + s * part_stride
        // Lane pairs (V = 2) or quads (V = 1) exchange rows, so a lane handles four neighbouring
        // columns of a row: two rows per lane and register group (V = 2), or one (V = 1).
        const bool resid = ep.kind == EP_RESID;
        const bool rd_delta = resid ? ep.delta_mode == 2 : ep.kind == EP_SKIP && ep.delta_mode == 1;
        float* const hdst = ep.kind == EP_PARTIAL ? ep.h + (long)split * ep.part_stride : ep.h;
        const float* const hsrc = ep.hin ? ep.hin : ep.h;
        groups([&](auto jc, auto vc, int n) {
            constexpr int J = decltype(jc)::value, V = decltype(vc)::value;
            constexpr int RL = V;                     // rows per lane and register group
            constexpr int QB = 2;                     // register groups per load batch
            const int n4 = V == 2 ? n - 2 * (l & 1) : n - lq;  // first of the lane's four columns
            const int nl = min(n4, g.N - 4);          // clamped: every load stays inside
            float b[V];
#pragma unroll
            for (int v = 0; v < V; ++v) b[v] = ep.bias && split == 0 && n < g.N ? ep.bias[n + v] : 0.f;
            // row of the lane's w-th row in register group q of block i
            auto lane_row = [&](int i, int q, int w) { return row_of(i, q) + (V == 2 ? 2 * w + (l & 1) : lq); };
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q0 = 0; q0 < 4; q0 += QB) {
                    f32x4 hv[QB][RL], dv[QB][RL], gt[QB][RL], zv[QB][RL];
#pragma unroll
                    for (int q = 0; q < QB; ++q)
#pragma unroll
                        for (int w = 0; w < RL; ++w) {
                            const int row = min(lane_row(i, q0 + q, w), g.M - 1);
                            const long idx = (long)row * ep.d + nl;
                            hv[q][w] = resid ? *(const f32x4*)(hsrc + idx) : f32x4{0.f, 0.f, 0.f, 0.f};
                            zv[q][w] = ep.z ? *(const f32x4*)(ep.z + idx) : f32x4{0.f, 0.f, 0.f, 0.f};
                            dv[q][w] = rd_delta ? *(const f32x4*)(ep.delta + idx) : f32x4{0.f, 0.f, 0.f, 0.f};
                            gt[q][w] = ep.gate ? *(const f32x4*)(ep.gate + (long)sample_of(row) * ep.gate_ld + nl)
                                               : f32x4{1.f, 1.f, 1.f, 1.f};
                        }
#pragma unroll
                    for (int q = 0; q < QB; ++q) {
                        f32x4 x[RL];
                        if constexpr (V == 2) {
                            // rows 2 w (even lanes) and 2 w + 1 (odd lanes): own pair and the neighbour's
#pragma unroll
                            for (int w = 0; w < 2; ++w) {
                                const int r = (q0 + q) * 4 + 2 * w;
#pragma unroll
                                for (int v = 0; v < 2; ++v) {
                                    const float e = acc[i][J + v][r] + b[v], o = acc[i][J + v][r + 1] + b[v];
                                    const float pe = __uint_as_float(quad_xor1(__float_as_uint(e)));
                                    const float po = __uint_as_float(quad_xor1(__float_as_uint(o)));
                                    x[w][v] = (l & 1) ? po : e;
                                    x[w][2 + v] = (l & 1) ? o : pe;
                                }
                            }
                        } else {
                            uint32_t t[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u) t[u] = __float_as_uint(acc[i][J][(q0 + q) * 4 + u] + b[0]);
                            quad_transpose(t, l);
#pragma unroll
                            for (int u = 0; u < 4; ++u) x[0][u] = __uint_as_float(t[u]);
                        }
#pragma unroll
                        for (int w = 0; w < RL; ++w) {
                            const int row = lane_row(i, q0 + q, w);
                            if (row >= g.M || n4 >= g.N) continue;
                            const long idx = (long)row * ep.d + n4;
                            f32x4 xx = x[w], hn;
                            if (ep.gate) xx = xx * gt[q][w];
                            const f32x4 dn = dv[q][w] + xx;
                            hn = resid ? hv[q][w] + xx : rd_delta ? dn : xx;
                            if (!ep.z) {
                                *(f32x4*)(hdst + idx) = hn;
                            } else {
                                const int tok = row - sample_of(row) * ep.ntok;
                                if (tok >= ep.r0 && tok < ep.r1) *(f32x4*)(ep.z + idx) = zv[q][w] * ep.alpha - hn * ep.beta;
                            }
                            if (resid && ep.delta_mode == 1) *(f32x4*)(ep.delta + idx) = xx;
                            if (resid && ep.delta_mode == 2) *(f32x4*)(ep.delta + idx) = dn;
                            if (ep.hcopy) {
                                const float t[4] = {hn[0], hn[1], hn[2], hn[3]};
                                store_bf16x4((bf16*)ep.hcopy + idx, t);
                            }
                        }
                    }
                }
        });
    }
}

// --------------------------------------------------------------------------- loads

// 16 bytes a lane from buffer r at voff + soff to LDS byte address lds + 16 lane (voff out of the
// descriptor's range: zeros).  Counted in vmcnt; the caller waits.  m0 (the LDS address) is used by
// nothing else in these kernels.
__device__ __forceinline__ void dma16(unsigned lds, unsigned voff, u32x4 r, unsigned soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(voff), "s"(r), "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory");
}
template <int N>
__device__ __forceinline__ void vm_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// workgroup barrier without the waits of __syncthreads (outstanding loads stay in flight)
__device__ __forceinline__ void raw_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// buffer descriptor as four scalars (nothing is in range when bytes = 0)
__device__ __forceinline__ u32x4 buf_desc(const void* base, unsigned bytes) {
    const uint64_t p = (uint64_t)base;
    u32x4 r;
    r[0] = __builtin_amdgcn_readfirstlane((unsigned)p);
    r[1] = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32));
    r[2] = bytes;
    r[3] = 0x00020000;
    return r;
}

}  // namespace sgd
