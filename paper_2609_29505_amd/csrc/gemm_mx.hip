// Products of microscaled rows: C = A . W^T with A in e4m3 or e2m1, W in e2m1, a power-of-two scale per
// 32 columns of either (mx.h), fp32 accumulation, and the bf16 GEMM's epilogues.
//
// Matrix instructions: v_mfma_scale_f32_32x32x64_f8f6f4 takes the scales of a lane's 32-column block with
// the operands.  A lane of an e2m1 operand holds columns 32 h .. 32 h + 31 of its row (h = lane / 32) in 16 bytes;
// one of an e4m3 operand columns 16 h .. and 32 + 16 h .. in twice 16 bytes; the scale it carries is that
// of block h either way.  With both operands in e2m1 an instruction takes as long as a bf16 one of 16
// columns, so a k tile of 256 columns (128 bytes a row) has the LDS traffic and the matrix-core time
// of the bf16 kernels' 64; with A in e4m3 it takes twice that, and 128 columns make the k tile (128
// bytes of A, 64 of W).
//
// Sums: with A in e2m1 products are exact and the sums right to fp32 rounding (2.4e-8 to 3e-8 of the result
// measured).  With A in e4m3 the instruction adds the products of eight neighbouring columns aligned to the largest
// exponent among them, each cut 13 bits below it (toward zero), and the groups and steps in fp32: exact where a group's
// elements of A lie within eight binades, else off by less than 7 2^-13 of a group's largest product.  Of
// sqrt(sum (a w)^2) measured: rows quantised from normal values 4e-6 rms, 4e-5 at most; codes from all of e4m3 4.5e-5 and
// 3e-4, below a bf16 output's rounding (2e-3).  fp32 output keeps what the instruction gives.
//
// Three kernels.  gemm_mx_pp_kernel and gemm_mx_pk_kernel are the two schedules of gemm_bf16.hip (large
// tiles shared by two wave groups half a phase apart; small tiles whose groups split K) with the scales
// as one more piece of a stage; gemm_mx_rows_kernel takes up to 16 rows of A, where the
// time is that of reading W once.
#include <algorithm>

#include "common.h"
#include "gemm_common.h"
#include "kernels.h"
#include "mx.h"
#include "tile_order.h"

namespace sgd {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// 4 bytes a lane to LDS, as dma16
__device__ __forceinline__ void dma4(unsigned lds, unsigned voff, u32x4 r, unsigned soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(voff), "s"(r), "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory");
}

// What a k tile is for a format of A
template <int FA> struct MxK {
    static constexpr bool FP8 = FA == MX_FP8;
    static constexpr int KE = FP8 ? 128 : 256;    // columns
    static constexpr int WB = KE / 2;             // bytes of a W row (128 of an A row)
    static constexpr int STEPS = KE / 64;         // matrix steps
    static constexpr int SB = KE / 32;            // scale bytes of a row
    static constexpr int CBSZ = FP8 ? 0 : 4;      // the instruction's code of A's format (W: 4)
    static constexpr int BROWS = 8192 / WB;       // W rows that 512 lanes load at once
    // LDS position of 16-byte chunk c of row r, so that the reads of 16 consecutive rows cover the 64 banks once
    __device__ static __forceinline__ int apos(int r, int c) { return c ^ ((r >> 1) & 7); }
    __device__ static __forceinline__ int wpos(int r, int c) { return FP8 ? c ^ ((r >> 2) & 3) : c ^ ((r >> 1) & 7); }
};

// the scale bytes of a lane's blocks (2 q + h for steps q) as the bytes q of one word
template <int FA>
__device__ __forceinline__ int pick_scales(const char* at, int half) {
    if constexpr (FA == MX_FP8) {
        const uint32_t v = *(const uint32_t*)at;
        return (int)__builtin_amdgcn_perm(v, v, half ? 0x03010301u : 0x02000200u);
    } else {
        const u32x2 v = *(const u32x2*)at;
        return (int)__builtin_amdgcn_perm(v[1], v[0], half ? 0x07050301u : 0x06040200u);
    }
}

// A lane's operand: 16 bytes (e2m1) or two pieces of 16 (e4m3); the instruction's upper half is not read for e2m1
template <int FA> using MxFrag = std::conditional_t<FA == MX_FP8, i32x8, i32x4>;
__device__ __forceinline__ i32x8 widen(const i32x8& x) { return x; }
__device__ __forceinline__ i32x8 widen(const i32x4& x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }
template <int FA, int Q>
__device__ __forceinline__ f32x16 mx_mfma(const MxFrag<FA>& a, const i32x4& b, const f32x16& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(a), widen(b), c, MxK<FA>::CBSZ, 4, Q, sa, Q, sb);
}
// step q's A fragment: chunk 2 q + half, or 4 q + half and 4 q + 2 + half; f: place of chunk half
template <int FA>
__device__ __forceinline__ MxFrag<FA> read_frag(const char* lds, unsigned f, int q, int off) {
    if constexpr (FA == MX_FP8)
        return __builtin_shufflevector(*(const i32x4*)(lds + (f ^ (q * 64)) + off), *(const i32x4*)(lds + (f ^ (q * 64 + 32)) + off), 0,
                                       1, 2, 3, 4, 5, 6, 7);
    else return *(const i32x4*)(lds + (f ^ (q * 32)) + off);
}

// What the epilogue of a kind reads, the kind a compile-time constant
template <int KIND>
__device__ __forceinline__ EpiParams mx_epilogue(const EpiParams& p) {
    EpiParams e;
    e.kind = KIND;
    e.bias = p.bias;
    if constexpr (KIND == EP_PARTIAL) { e.h = p.h; e.d = p.d; }
    else { e.out = p.out; e.ldo = p.ldo; e.act = p.act; e.F = p.F; }
    return e;
}

// --------------------------------------------------------------------------- large tiles
//
// 8192 x 12288 x 4096 in e2m1 213-223 us (3.7-3.9 PFLOP/s): six rounds of 256 x 256 tiles, each 16 k tiles of 1.6 us and some 8.5 us
// of start and epilogue (fitted over K 1024 to 8192).  A k tile moves 64 KB into the LDS and 192 KB out of it, 2048 clocks at 128 bytes,
// and its matrix instructions take 2048 clocks: either alone would be 1.0 us, and the phases, of which one reads two
// thirds of the fragments, wait for each other.  1024 x 24576 x 4096 gated, A in e4m3, 79-85 us (2.5 PFLOP/s).

template <int FA, int BM_, int BN_, int WGM_, int WGN_, int ST_ = 2>
struct MxPPCfg {
    using K = MxK<FA>;
    static constexpr int FMT = FA, BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, ST = ST_, NT = 512, NW = 8;
    static constexpr int BH = BM / 2, HP = BH / 64;      // rows and load parts (64 rows) of each half
    static constexpr int RW = BH / WGM;                  // a wave's rows of each half
    static constexpr int CB = RW / 32, TM = 2 * CB;      // MFMA row blocks per half, per wave
    static constexpr int WN = BN / WGN, TN = WN / 32;
    static constexpr int BP = (BN + K::BROWS - 1) / K::BROWS, BL = BP / 2;  // W parts per tile; those loaded in phase 1
    static constexpr int A_HALF = BH * 128, A_STAGE = BM * 128, B_STAGE = BP * 8192;
    static constexpr int SC = ((BM + BN) * K::SB + 2047) / 2048, S_STAGE = SC * 2048;  // scales: A's rows, then W's
    static constexpr int B_LDS = ST * A_STAGE, S_LDS = B_LDS + ST * B_STAGE, LDS_BYTES = S_LDS + ST * S_STAGE;
    __device__ static __forceinline__ int block_row(int wm, int i) { return (i / CB) * BH + wm * RW + (i % CB) * 32; }
    static_assert(WGM * WGN == NW && RW % 32 == 0 && WN % 32 == 0 && BH % 64 == 0, "wave tile");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS");
};

// A wave's source of scale words: A's or W's rows
struct MxScaleSrc { const char* base; unsigned bytes; int rows; };
__device__ __forceinline__ MxScaleSrc mx_scale_source(bool of_a, const GemmArgs& g, const MxScales& s) {
    const unsigned chunks = (unsigned)(g.K + 255) / 256 * 8;
    MxScaleSrc r;
    r.base = (const char*)(of_a ? s.a : s.w);
    r.rows = of_a ? g.M : g.N;
    r.bytes = chunks * (unsigned)r.rows;
    return r;
}

// A tile's sources: A from its first row on, W whole
struct MxTileSrc {
    const char *a, *w;
    unsigned na, nw;            // bytes in range
    int KT;                     // k tiles
    unsigned lasta, lastw;      // 16-byte chunks of a row in the last k tile
};
template <int FA>
__device__ __forceinline__ MxTileSrc mx_source(const GemmArgs& g, int m0, int bm) {
    using K = MxK<FA>;
    const long ra = FA == MX_FP8 ? g.K : g.K / 2, rw = g.K / 2;  // bytes of a row
    MxTileSrc t;
    t.a = (const char*)g.A0 + m0 * ra;
    t.na = (unsigned)(min(g.M - m0, bm) * ra);
    t.w = (const char*)g.B;
    t.nw = (unsigned)(g.N * rw);
    t.KT = (g.K + K::KE - 1) / K::KE;
    const int rest = g.K - (t.KT - 1) * K::KE;
    t.lasta = rest / (FA == MX_FP8 ? 16 : 32);
    t.lastw = rest / 32;
    return t;
}
constexpr unsigned kMxOob = 0xFFFFFF00u;

// The scale word that lane i of load p brings: 4 bytes of a row of A (i below its rows) or of W
template <class C>
__device__ __forceinline__ unsigned mx_scale_off(const GemmArgs& g, const EpiParams& ep, int m0, int tn, int i) {
    constexpr int PER = C::K::SB / 4;
    const int r = i / PER, sub = i % PER;
    if (r < C::BM) {
        const int row = m0 + r;
        return row < g.M ? (unsigned)row * 8u + sub * 4 : kMxOob;
    }
    if (r >= C::BM + C::BN) return kMxOob;
    const long row = weight_row<C>(ep, g.N / 2, tn, r - C::BM);
    return row < g.N ? (unsigned)row * 8u + sub * 4 : kMxOob;
}
// byte offset of k tile t in a scale array of `rows` rows
template <int FA>
__device__ __forceinline__ unsigned mx_scale_tile(int t, int rows) {
    return FA == MX_FP8 ? (unsigned)(t >> 1) * (unsigned)rows * 8u + (t & 1) * 4 : (unsigned)t * (unsigned)rows * 8u;
}

template <class C, int KIND>
__global__ __launch_bounds__(C::NT, 2) void gemm_mx_pp_kernel(GemmArgs g, EpiParams params, MxScales sc) {
    const EpiParams ep = mx_epilogue<KIND>(params);
    using K = typename C::K;
    constexpr int FA = C::FMT;
    __shared__ __attribute__((aligned(1024))) char lds[C::LDS_BYTES];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nt_m = (g.M + C::BM - 1) / C::BM, nt_n = (g.N + C::BN - 1) / C::BN;
    int tm, tn;
    tile_at(tile_position((int)blockIdx.x, nt_m * nt_n), nt_m, nt_n, g.band, tm, tn);
    const int m0 = tm * C::BM;
    const MxTileSrc src = mx_source<FA>(g, m0, C::BM);
    const int KT = src.KT;

    // load parts: A 64 rows of 8 chunks; W 64 rows of 8 or 128 of 4
    const int arow = wave * 8 + (lane >> 3), achunk = K::apos(arow, lane & 7);
    constexpr int WC = K::WB / 16;
    const int wrow = wave * (64 / WC) + lane / WC, wchunk = K::wpos(wrow, lane % WC);
    const int ra = FA == MX_FP8 ? g.K : g.K / 2, rw = g.K / 2;
    // Part 0; A's others follow at even distances, and W's do where a part is whole waves' columns.  Rows past M or N
    // are past the buffer's range
    constexpr bool EVEN = K::BROWS % C::WN == 0;
    const unsigned aoff = (unsigned)(arow * ra + achunk * 16);
    const int astep = 64 * ra, bstep = (int)(weight_row<C>(ep, g.N / 2, tn, K::BROWS) - weight_row<C>(ep, g.N / 2, tn, 0)) * rw;
    unsigned boff[EVEN ? 1 : C::BP];
#pragma unroll
    for (int p = 0; p < (EVEN ? 1 : C::BP); ++p) {
        const int r = p * K::BROWS + wrow;
        boff[p] = r < C::BN ? (unsigned)(weight_row<C>(ep, g.N / 2, tn, r) * rw + wchunk * 16) : kMxOob;
    }
    unsigned soff[C::SC];
#pragma unroll
    for (int p = 0; p < C::SC; ++p) soff[p] = mx_scale_off<C>(g, ep, m0, tn, p * 512 + tid);
    // waves of A's rows and of W's rows of scales (a wave's 64 words belong to one of them)
    MxScaleSrc ssrc[C::SC];
#pragma unroll
    for (int p = 0; p < C::SC; ++p) ssrc[p] = mx_scale_source((p * 512 + wave * 64) / (K::SB / 4) < C::BM, g, sc);
    const unsigned lw = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * 1024;
    const unsigned ls = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds + C::S_LDS + wave * 256;
    // tiles at or past K load zeros, as do the chunks past K of the last one
    auto load_a = [&](int t, int stage, int h) {
        const bool in = t < KT, last = t == KT - 1 && (unsigned)achunk >= src.lasta;
        const u32x4 r = buf_desc(src.a, in ? src.na : 0);
        int step = astep;
        asm volatile("" : "+s"(step));  // an addition a load instead of a register held for each
#pragma unroll
        for (int i = 0; i < C::HP; ++i)
            dma16(lw + stage * C::A_STAGE + h * C::A_HALF + i * 8192, last ? kMxOob : aoff + (h * C::HP + i) * step, r, in ? t * 128 : 0);
    };
    auto load_b = [&](int t, int stage, auto from, auto to) {
        const bool in = t < KT, last = t == KT - 1 && (unsigned)wchunk >= src.lastw;
        const u32x4 r = buf_desc(src.w, in ? src.nw : 0);
        int step = bstep;
        asm volatile("" : "+s"(step));
#pragma unroll
        for (int p = decltype(from)::value; p < decltype(to)::value; ++p)
            dma16(lw + C::B_LDS + stage * C::B_STAGE + p * 8192, last ? kMxOob : EVEN ? boff[0] + p * step : boff[EVEN ? 0 : p], r, in ? t * K::WB : 0);
    };
    auto load_s = [&](int t, int stage) {
        const bool in = t < KT;
#pragma unroll
        for (int p = 0; p < C::SC; ++p) {
            dma4(ls + stage * C::S_STAGE + p * 2048, soff[p], buf_desc(ssrc[p].base, in ? ssrc[p].bytes : 0),
                 in ? mx_scale_tile<FA>(t, ssrc[p].rows) : 0);
        }
    };

    const int wm = wave / C::WGN, wn = wave % C::WGN, wn0 = wn * C::WN;
    const int lrow = lane & 31, lhalf = lane >> 5;
    // fragment addresses of step 0; step q's chunk is XORed in (the swizzle is an XOR too), which costs an
    // instruction instead of a register held for every step
    const unsigned fa = (unsigned)((wm * C::RW + lrow) * 128 + (K::apos(lrow, lhalf) << 4));
    const unsigned fb = (unsigned)(C::B_LDS + (wn0 + lrow) * K::WB + (K::wpos(lrow, lhalf) << 4));
    const char* const fsa = lds + C::S_LDS + (wm * C::RW + lrow) * K::SB;
    const char* const fsb = lds + C::S_LDS + (C::BM + wn0 + lrow) * K::SB;
    f32x16 acc[C::TM][C::TN];
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    MxFrag<FA> af[C::CB][K::STEPS];
    i32x4 bfr[C::TN][K::STEPS];
    int sa[C::TM], sb[C::TN];
    auto read_a = [&](int stage, int h) {
        unsigned f = fa;
        asm volatile("" : "+v"(f));
#pragma unroll
        for (int q = 0; q < K::STEPS; ++q)
#pragma unroll
            for (int i = 0; i < C::CB; ++i) af[i][q] = read_frag<FA>(lds, f, q, stage * C::A_STAGE + h * C::A_HALF + i * 4096);
    };
    auto read_b = [&](int stage) {
#pragma unroll
        for (int j = 0; j < C::TN; ++j) sb[j] = pick_scales<FA>(fsb + stage * C::S_STAGE + j * 32 * K::SB, lhalf);
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
            sa[i] = pick_scales<FA>(fsa + stage * C::S_STAGE + ((i / C::CB) * C::BH + (i % C::CB) * 32) * K::SB, lhalf);
        unsigned f = fb;
        asm volatile("" : "+v"(f));
#pragma unroll
        for (int q = 0; q < K::STEPS; ++q)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) bfr[j][q] = *(const i32x4*)(lds + (f ^ (q * 32)) + stage * C::B_STAGE + j * 32 * K::WB);
    };
    auto mfmas = [&](int h) {
        static_for<K::STEPS>([&](auto qc) {
            constexpr int q = decltype(qc)::value;
#pragma unroll
            for (int i = 0; i < C::CB; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j)
                    acc[h * C::CB + i][j] = mx_mfma<FA, q>(af[i][q], bfr[j][q], acc[h * C::CB + i][j], sa[h * C::CB + i], sb[j]);
        });
    };
    // end of a phase's reads: the fragments are in registers before the other group may refill
    auto turn = [&] {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        raw_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr IntC<0> B0{};
    constexpr IntC<C::BL> BLO{};
    constexpr IntC<C::BP> B1{};
    // Load order per tile: A half 0, the scales and the first BL W parts (phase 1 of tile t - ST), the other W
    // parts and A half 1 (phase 0 of tile t - ST + 1).  All scales are read in phase 0.  Before phase 1 of tile
    // t is read, at most the loads issued after its A half 1 may be outstanding: ST - 1 tiles' worth; before
    // phase 0 of tile t, those after its W parts: its A half 1, ST - 1 phases 1 and ST - 2 phases 0.
    constexpr int L1 = C::HP + C::SC + C::BL, L0 = C::BP - C::BL + C::HP;  // loads of phases 1 and 0
    constexpr int W0 = (C::ST - 1) * (L0 + L1), W1 = C::HP + (C::ST - 1) * L1 + (C::ST - 2) * L0;
    static_assert(W0 < 64, "vmcnt");
    static_for<C::ST - 1>([&](auto stc) {
        constexpr int s = decltype(stc)::value;
        load_a(s, s, 0);
        load_s(s, s);
        load_b(s, s, B0, B1);
        load_a(s, s, 1);
    });
    load_a(C::ST - 1, C::ST - 1, 0);
    load_s(C::ST - 1, C::ST - 1);
    load_b(C::ST - 1, C::ST - 1, B0, BLO);
    vm_wait<W1>();
    raw_barrier();
    const bool late = wave >= 4;  // the second group runs half a phase behind
    if (late) raw_barrier();
    auto tile = [&](int t, auto stc) {
        constexpr int s = decltype(stc)::value, prev = (s + C::ST - 1) % C::ST;
        __builtin_amdgcn_sched_barrier(0);
        read_b(s);
        read_a(s, 0);
        load_b(t + C::ST - 1, prev, BLO, B1);
        load_a(t + C::ST - 1, prev, 1);
        vm_wait<W0>();
        turn();
        mfmas(0);
        __builtin_amdgcn_sched_barrier(0);
        raw_barrier();
        __builtin_amdgcn_sched_barrier(0);
        read_a(s, 1);
        load_a(t + C::ST, s, 0);
        load_s(t + C::ST, s);
        load_b(t + C::ST, s, B0, BLO);
        vm_wait<W1>();
        turn();
        mfmas(1);
        __builtin_amdgcn_sched_barrier(0);
        raw_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int t = 0; t < KT; t += C::ST)
        static_for<C::ST>([&](auto stc) {
            if (t + decltype(stc)::value < KT) tile(t + decltype(stc)::value, stc);
        });
    if (!late) raw_barrier();
    vm_wait<0>();
    // the epilogue's arguments are read again here instead of being held across the main loop
    const char __attribute__((address_space(4)))* args =
        (const char __attribute__((address_space(4)))*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    constexpr int EP_AT = (sizeof(GemmArgs) + alignof(EpiParams) - 1) / alignof(EpiParams) * alignof(EpiParams);
    epilogue<C>(acc, *(const GemmArgs*)(const char*)args, mx_epilogue<KIND>(*(const EpiParams*)(const char*)(args + EP_AT)), m0, tn,
                wm, wn, 0);
}

// --------------------------------------------------------------------------- K-group kernel
//
// For few or ragged tiles, where the chip is not full and the time is the latency of a tile's chain of k tiles: two groups
// of four waves halve it.

template <int FA, int BM_, int BN_, int S_>
struct MxPKCfg {
    using K = MxK<FA>;
    static constexpr int FMT = FA, BM = BM_, BN = BN_, S = S_, NT = 512;
    static constexpr int TMW = BM / 64, TN = BN / 64, WN = BN / 2;  // a wave's MFMA blocks, columns
    static constexpr int TM = 1;                                    // row blocks per wave in the epilogue
    static constexpr int SC = ((BM + BN) * K::SB + 1023) / 1024, S_BYTES = SC * 1024;
    static constexpr int AP = BM / 32, BP = BN * K::WB / 4096, P = AP + BP + SC;  // loads per wave and k tile
    static constexpr int SLOTS = K::STEPS * TMW * TN;                // matrix instructions of a k tile
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * K::WB, STAGE = A_BYTES + B_BYTES + S_BYTES;
    static constexpr int LDS_BYTES = 2 * S * STAGE;
    // two-block waves: group g finishes row block g of its wave row (row index wm * 2 + g)
    __device__ static __forceinline__ int block_row(int w, int) { return w * 32; }
    static_assert((TMW == 1 || TMW == 2) && (S - 1) * P < 64 && BN * K::WB % 4096 == 0, "k-group tile");
    static_assert(LDS_BYTES <= 160 * 1024 && LDS_BYTES >= BM * BN * 4, "LDS: stages, then the exchange");
};

template <class C, int KIND>
__global__ __launch_bounds__(C::NT, 2) void gemm_mx_pk_kernel(GemmArgs g, EpiParams params, MxScales sc) {
    const EpiParams ep = mx_epilogue<KIND>(params);
    using K = typename C::K;
    constexpr int FA = C::FMT;
    __shared__ __attribute__((aligned(1024))) char lds[C::LDS_BYTES];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = wave >> 2, gw = wave & 3;
    const int nt_m = (g.M + C::BM - 1) / C::BM, nt_n = (g.N + C::BN - 1) / C::BN;
    int tm, tn;
    tile_at(tile_position((int)blockIdx.x, nt_m * nt_n), nt_m, nt_n, g.band, tm, tn);
    const int m0 = tm * C::BM;
    const MxTileSrc src = mx_source<FA>(g, m0, C::BM);
    const int KT = src.KT;

    const int arow = gw * 8 + (lane >> 3), achunk = K::apos(arow, lane & 7);
    constexpr int WC = K::WB / 16, WR = 4 * (64 / WC);  // W chunks of a row, W rows of a part
    const int wrow = gw * (64 / WC) + lane / WC, wchunk = K::wpos(wrow, lane % WC);
    const int ra = FA == MX_FP8 ? g.K : g.K / 2, rw = g.K / 2;
    unsigned off[C::P];
    MxScaleSrc ssrc[C::SC];
#pragma unroll
    for (int p = 0; p < C::AP; ++p) off[p] = (unsigned)((p * 32 + arow) * ra + achunk * 16);
#pragma unroll
    for (int p = 0; p < C::BP; ++p) {
        const long row = weight_row<C>(ep, g.N / 2, tn, p * WR + wrow);
        off[C::AP + p] = row < g.N ? (unsigned)(row * rw + wchunk * 16) : kMxOob;
    }
#pragma unroll
    for (int p = 0; p < C::SC; ++p) {
        off[C::AP + C::BP + p] = mx_scale_off<C>(g, ep, m0, tn, p * 256 + gw * 64 + lane);
        ssrc[p] = mx_scale_source((p * 256 + gw * 64) / (K::SB / 4) < C::BM, g, sc);
    }
    const unsigned l0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds + grp * (C::S * C::STAGE);
    // the group's i-th k tile into stage i % S; tiles at or past K load zeros
    struct Src { u32x4 ra, rb; unsigned sa, sb; int t; bool in, cuta, cutw; };
    auto source = [&](int i) {
        Src c;
        c.t = 2 * i + grp;
        c.in = c.t < KT;
        c.ra = buf_desc(src.a, c.in ? src.na : 0);
        c.rb = buf_desc(src.w, c.in ? src.nw : 0);
        c.sa = c.in ? c.t * 128 : 0;
        c.sb = c.in ? c.t * K::WB : 0;
        c.cuta = c.t == KT - 1 && (unsigned)achunk >= src.lasta;
        c.cutw = c.t == KT - 1 && (unsigned)wchunk >= src.lastw;
        return c;
    };
    auto load = [&](const Src& c, unsigned l, int p) {
        if (p < C::AP) {
            dma16(l + gw * 1024 + p * 4096, c.cuta ? kMxOob : off[p], c.ra, c.sa);
        } else if (p < C::AP + C::BP) {
            dma16(l + gw * 1024 + C::A_BYTES + (p - C::AP) * 4096, c.cutw ? kMxOob : off[p], c.rb, c.sb);
        } else {
            const int s = p - C::AP - C::BP;
            dma4(l + gw * 256 + C::A_BYTES + C::B_BYTES + s * 1024, off[p], buf_desc(ssrc[s].base, c.in ? ssrc[s].bytes : 0),
                 c.in ? mx_scale_tile<FA>(c.t, ssrc[s].rows) : 0);
        }
    };

    const int wm = gw >> 1, wn = gw & 1;
    const int lrow = lane & 31, lhalf = lane >> 5;
    const unsigned gl = grp * (C::S * C::STAGE);
    const unsigned fa = gl + (wm * (C::BM / 2) + lrow) * 128 + (K::apos(lrow, lhalf) << 4);
    const unsigned fb = gl + C::A_BYTES + (wn * C::WN + lrow) * K::WB + (K::wpos(lrow, lhalf) << 4);
    const char* const fsa = lds + gl + C::A_BYTES + C::B_BYTES + (wm * (C::BM / 2) + lrow) * K::SB;
    const char* const fsb = lds + gl + C::A_BYTES + C::B_BYTES + (C::BM + wn * C::WN + lrow) * K::SB;
    f32x16 acc[C::TMW][C::TN];
#pragma unroll
    for (int i = 0; i < C::TMW; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

#pragma unroll
    for (int s = 0; s < C::S; ++s) {
        const Src c = source(s);
#pragma unroll
        for (int p = 0; p < C::P; ++p) load(c, l0 + s * C::STAGE, p);
    }
    constexpr int W = (C::S - 1) * C::P;  // the next tile has landed; those after it may be in flight
    vm_wait<W>();
    raw_barrier();
    if (grp) raw_barrier();
    const int steps = (KT + 1) / 2;  // the same for both groups: barriers match
    int stage = 0;
    for (int i = 0; i < steps; ++i) {
        const int so = stage * C::STAGE;
        MxFrag<FA> af[C::TMW][K::STEPS];
        i32x4 bfr[C::TN][K::STEPS];
        int sa[C::TMW], sb[C::TN];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < C::TMW; ++x) sa[x] = pick_scales<FA>(fsa + so + x * 32 * K::SB, lhalf);
#pragma unroll
        for (int x = 0; x < C::TN; ++x) sb[x] = pick_scales<FA>(fsb + so + x * 32 * K::SB, lhalf);
#pragma unroll
        for (int q = 0; q < K::STEPS; ++q) {
#pragma unroll
            for (int x = 0; x < C::TMW; ++x) af[x][q] = read_frag<FA>(lds, fa, q, so + x * 4096);
#pragma unroll
            for (int x = 0; x < C::TN; ++x) bfr[x][q] = *(const i32x4*)(lds + (fb ^ (q * 32)) + so + x * 32 * K::WB);
        }
        const Src c = source(i + C::S);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        raw_barrier();
        __builtin_amdgcn_sched_barrier(0);
        // the loads that refill the stage just read go between the matrix instructions
        static_for<K::STEPS>([&](auto qc) {
            constexpr int q = decltype(qc)::value;
#pragma unroll
            for (int x = 0; x < C::TMW; ++x)
#pragma unroll
                for (int y = 0; y < C::TN; ++y) {
                    acc[x][y] = mx_mfma<FA, q>(af[x][q], bfr[y][q], acc[x][y], sa[x], sb[y]);
                    const int slot = (q * C::TMW + x) * C::TN + y;
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int p = slot * C::P / C::SLOTS; p < (slot + 1) * C::P / C::SLOTS; ++p) load(c, l0 + so, p);
                    __builtin_amdgcn_sched_barrier(0);
                }
        });
        vm_wait<W>();
        __builtin_amdgcn_sched_barrier(0);
        raw_barrier();
        stage = stage + 1 == C::S ? 0 : stage + 1;
    }
    if (!grp) raw_barrier();
    vm_wait<0>();  // the loads past K have written their zeros before LDS is used for the exchange
    raw_barrier();
    // exchange: register group of four of block (x, y), register quad q, of wave gw: 1 KB a wave
    f32x4* const ex = (f32x4*)lds;
    auto slot_of = [&](int y, int q, int half) { return (((half * 4 + gw) * C::TN + y) * 4 + q) * 64 + lane; };
    f32x16 sum[1][C::TN];
    if constexpr (C::TMW == 2) {
#pragma unroll
        for (int y = 0; y < C::TN; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 o;  // the other group's row block
#pragma unroll
                for (int u = 0; u < 4; ++u) o[u] = grp ? acc[0][y][q * 4 + u] : acc[1][y][q * 4 + u];
                ex[slot_of(y, q, grp)] = o;
            }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < C::TN; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 o = ex[slot_of(y, q, grp ^ 1)];
#pragma unroll
                for (int u = 0; u < 4; ++u) sum[0][y][q * 4 + u] = (grp ? acc[1][y][q * 4 + u] : acc[0][y][q * 4 + u]) + o[u];
            }
    } else {
        if (grp) {
#pragma unroll
            for (int y = 0; y < C::TN; ++y)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 o;
#pragma unroll
                    for (int u = 0; u < 4; ++u) o[u] = acc[0][y][q * 4 + u];
                    ex[slot_of(y, q, 0)] = o;
                }
        }
        __syncthreads();
        if (grp) return;
#pragma unroll
        for (int y = 0; y < C::TN; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 o = ex[slot_of(y, q, 0)];
#pragma unroll
                for (int u = 0; u < 4; ++u) sum[0][y][q * 4 + u] = acc[0][y][q * 4 + u] + o[u];
            }
    }
    const char __attribute__((address_space(4)))* args =
        (const char __attribute__((address_space(4)))*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    constexpr int EP_AT = (sizeof(GemmArgs) + alignof(EpiParams) - 1) / alignof(EpiParams) * alignof(EpiParams);
    epilogue<C>(sum, *(const GemmArgs*)(const char*)args, mx_epilogue<KIND>(*(const EpiParams*)(const char*)(args + EP_AT)), m0, tn,
                wm * C::TMW + (C::TMW == 2 ? grp : 0), wn, 0);
}

// --------------------------------------------------------------------------- few rows
//
// Up to 16 rows of A: W is streamed once from HBM, straight into registers, so W's rows are the rows of the
// matrix instruction (16x16x128: a lane holds 32 columns of W row lane % 16) and A's rows its columns.  A
// workgroup finishes 16 output columns (gated: 16 gate and their 16 up columns); its eight waves
// take alternate 128-column steps, each with UN of them in flight, and their sums meet in LDS in
// wave order.  A's rows come from the L2.  One row of 24576 x 4096 gated 12.3 us, 4.3 TB/s.

template <int FA>
__device__ __forceinline__ f32x4 mx_mfma16(const i32x4& w, const i32x8& a, const f32x4& c, int sw, int sa) {
    const i32x8 ww = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ww, a, c, 4, MxK<FA>::CBSZ, 0, sw, 0, sa);
}

template <int FA, int G>  // G: column groups of W (2: gate and up)
__global__ __launch_bounds__(512) void gemm_mx_rows_kernel(GemmArgs g, EpiParams ep, MxScales sc) {
    constexpr int NWV = 8, UN = 4;
    __shared__ f32x4 part[NWV][G][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l16 = lane & 15, lg = lane >> 4;
    const int nout = G == 2 ? ep.F : g.N;
    const int n0 = blockIdx.x * 16;
    const int steps = (g.K + 127) / 128;
    const long rw = g.K / 2, ra = FA == MX_FP8 ? g.K : g.K / 2;
    const bool row_in = l16 < g.M;
    const char *wp[G];
    const uint8_t* swp[G];
    bool col_in = n0 + l16 < nout;
#pragma unroll
    for (int j = 0; j < G; ++j) {
        const long n = (long)min(n0 + l16, nout - 1) + (j ? ep.F : 0);
        wp[j] = (const char*)g.B + n * rw + lg * 16;
        swp[j] = sc.w + n * 8 + lg;
    }
    const char* const ap = (const char*)g.A0 + (row_in ? l16 : 0) * ra;
    const uint8_t* const sap = sc.a + (long)(row_in ? l16 : 0) * 8 + lg;
    const long swc = (long)g.N * 8, sac = (long)g.M * 8;  // bytes of a chunk of scales
    f32x4 acc[G];
#pragma unroll
    for (int j = 0; j < G; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const i32x4 zero = {0, 0, 0, 0};
    for (int s0 = wave; s0 < steps; s0 += NWV * UN) {
        i32x4 w[UN][G], a0[UN], a1[UN];
        int sw[UN][G], sa[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int s = s0 + u * NWV;
            const bool in = s < steps && s * 128 + lg * 32 < g.K;  // K is whole 32-column blocks
            const long so = (long)(s >> 1) , sb = (s & 1) * 4;
#pragma unroll
            for (int j = 0; j < G; ++j) {
                w[u][j] = in && col_in ? __builtin_nontemporal_load((const i32x4*)(wp[j] + (long)s * 64)) : zero;
                sw[u][j] = in ? swp[j][so * swc + sb] : 0;
            }
            if constexpr (FA == MX_FP8) {
                // columns 16 lg .. and 64 + 16 lg ..
                const bool i0 = row_in && s < steps && s * 128 + lg * 16 < g.K, i1 = row_in && s < steps && s * 128 + 64 + lg * 16 < g.K;
                a0[u] = i0 ? *(const i32x4*)(ap + (long)s * 128 + lg * 16) : zero;
                a1[u] = i1 ? *(const i32x4*)(ap + (long)s * 128 + 64 + lg * 16) : zero;
            } else {
                a0[u] = in && row_in ? *(const i32x4*)(ap + (long)s * 64 + lg * 16) : zero;
                a1[u] = zero;
            }
            sa[u] = in ? sap[so * sac + sb] : 0;
        }
#pragma unroll
        for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int j = 0; j < G; ++j)
                acc[j] = mx_mfma16<FA>(w[u][j], __builtin_shufflevector(a0[u], a1[u], 0, 1, 2, 3, 4, 5, 6, 7), acc[j], sw[u][j], sa[u]);
    }
#pragma unroll
    for (int j = 0; j < G; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave) return;
    f32x4 v[G];
#pragma unroll
    for (int j = 0; j < G; ++j) {
        v[j] = part[0][j][lane];
#pragma unroll
        for (int w = 1; w < NWV; ++w) v[j] += part[w][j][lane];
    }
    // a lane holds columns n0 + 4 (lane / 16) .. + 3 of row lane % 16
    const int n = n0 + lg * 4;
    if (!row_in || n >= nout) return;
    if (ep.bias) {
#pragma unroll
        for (int j = 0; j < G; ++j) v[j] += *(const f32x4*)(ep.bias + n + (j ? ep.F : 0));
    }
    float o[4];
    with_act(ep.act, [&](auto actc) {
        constexpr int ACT = decltype(actc)::value;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = act_fn<ACT>(v[0][i]) * (G == 2 ? v[G - 1][i] : 1.f);
    });
    if (ep.kind == EP_PARTIAL) *(f32x4*)(ep.h + (long)l16 * ep.d + n) = f32x4{o[0], o[1], o[2], o[3]};
    else store_bf16x4((bf16*)ep.out + (long)l16 * ep.ldo + n, o);
}

// --------------------------------------------------------------------------- dispatch

namespace {
template <int FA> using X256x256 = MxPPCfg<FA, 256, 256, 2, 4>;
template <int FA> using X256x128 = MxPPCfg<FA, 256, 128, 4, 2, 3>;
template <int FA> using X128x256 = MxPPCfg<FA, 128, 256, 2, 4, 3>;
template <int FA> using X256x192 = MxPPCfg<FA, 256, 192, 4, 2>;
template <int FA> using X128x128 = MxPKCfg<FA, 128, 128, 2>;
template <int FA> using X128x64 = MxPKCfg<FA, 128, 64, 3>;
template <int FA> using X64x64 = MxPKCfg<FA, 64, 64, 4>;

// Block shape of a tile id, and what a tile takes with A in either format: us per k tile with the chip nearly
// empty and with every CU busy, and us for its start and epilogue.  Fitted to 520 products (17 to 8192 rows, 256 to
// 24576 columns, K 128 to 12288, weights cold), each timed with every tile: the choice made from them is
// within 0.1 % of the fastest tile on average and 5 % at worst (a first table, guessed from the bf16 kernels': 5 %
// off on 1024 rows of a gated 24576 x 4096 alone).  They rank tiles and are no model of a launch's time.
struct TileTime { double t0, t1, fix; };
struct Shape { int bm, bn; TileTime fp8, fp4; };
constexpr Shape kTiles[kMxTiles - 1] = {
    {256, 256, {0.630, 1.398, 11.2}, {0.798, 1.703, 9.7}},
    {256, 192, {0.702, 1.071, 8.8}, {0.813, 1.474, 8.9}},
    {256, 128, {0.611, 0.821, 6.3}, {0.717, 1.186, 6.4}},
    {128, 256, {0.596, 0.866, 6.3}, {0.809, 1.200, 6.4}},
    {128, 128, {0.348, 0.469, 6.3}, {0.466, 0.626, 6.9}},
    {128, 64, {0.205, 0.329, 5.6}, {0.242, 0.423, 5.6}},
    {64, 64, {0.176, 0.242, 5.0}, {0.182, 0.295, 5.0}},
};
}  // namespace

// Time (us) of a launch: n tiles are n / 256 whole rounds, one workgroup a CU, and a last one whose k tiles are
// faster the emptier it is.  Infinite where the epilogue cannot use the tile.
static double tile_cost(int tile, int fmt, const GemmArgs& g, const EpiParams& e) {
    const Shape& s = kTiles[tile - 1];
    if (e.kind == EP_GATED && g.N % s.bn) return 1e300;
    const TileTime& t = fmt == MX_FP8 ? s.fp8 : s.fp4;
    const long tiles = (long)((g.M + s.bm - 1) / s.bm) * ((g.N + s.bn - 1) / s.bn), ke = fmt == MX_FP8 ? 128 : 256;
    const double kt = (double)((g.K + ke - 1) / ke);
    auto round = [&](long n) { return kt * (t.t0 + (t.t1 - t.t0) * (double)n / 256.0) + t.fix; };
    return (double)(tiles / 256) * round(256) + (tiles % 256 ? round(tiles % 256) : 0.0);
}

// The kernel for few rows up to 16 of them (16 rows of a gated 24576 x 4096 17.8 us, 64 x 64 tiles 19.4; one row of
// 4096 x 12288 9.4 and 21.6), else the tile of least cost
int gemm_mx_tile(int fmt, const GemmArgs& g, const EpiParams& e) {
    if (g.M <= 16) return kMxTiles;
    int best = kMxTiles - 1;  // 64 x 64 takes every shape
    double best_t = 1e300;
    for (int tile = 1; tile < kMxTiles; ++tile) {
        const double t = tile_cost(tile, fmt, g, e);
        if (t < best_t) { best_t = t; best = tile; }
    }
    return best;
}

bool gemm_mx_shape_ok(int fmt, const GemmArgs& g, const EpiParams& e, int tile) {
    if (tile == 0) tile = gemm_mx_tile(fmt, g, e);
    // a launch has at most 2^32 threads
    const long nout = e.kind == EP_GATED ? e.F : g.N;
    if (tile == kMxTiles) return g.M <= 16 && nout < (1L << 27);
    const Shape& s = kTiles[tile - 1];
    return (e.kind != EP_GATED || g.N % s.bn == 0) &&
           (long)((g.M + s.bm - 1) / s.bm) * ((g.N + s.bn - 1) / s.bn) < (1L << 23);
}

template <class C> struct is_mx_pk : std::false_type {};
template <int FA, int BM, int BN, int S> struct is_mx_pk<MxPKCfg<FA, BM, BN, S>> : std::true_type {};

template <class C>
static hipError_t run_mx(const GemmArgs& g, const EpiParams& e, const MxScales& s, hipStream_t st) {
    const int nt_m = (g.M + C::BM - 1) / C::BM, nt_n = (g.N + C::BN - 1) / C::BN;
    GemmArgs ga = g;
    ga.band = tile_band(nt_m, nt_n, C::BM, C::BN);
    auto run = [&](auto kc) {
        constexpr int KIND = decltype(kc)::value;
        if constexpr (is_mx_pk<C>::value) gemm_mx_pk_kernel<C, KIND><<<nt_m * nt_n, C::NT, 0, st>>>(ga, e, s);
        else gemm_mx_pp_kernel<C, KIND><<<nt_m * nt_n, C::NT, 0, st>>>(ga, e, s);
    };
    switch (e.kind) {
        case EP_ACT: run(IntC<EP_ACT>{}); break;
        case EP_GATED: run(IntC<EP_GATED>{}); break;
        default: run(IntC<EP_PARTIAL>{}); break;
    }
    return hipGetLastError();
}

template <int FA>
static hipError_t run_mx_tile(const GemmArgs& g, const EpiParams& e, const MxScales& s, int tile, hipStream_t st) {
    switch (tile) {
        case 1: return run_mx<X256x256<FA>>(g, e, s, st);
        case 2: return run_mx<X256x192<FA>>(g, e, s, st);
        case 3: return run_mx<X256x128<FA>>(g, e, s, st);
        case 4: return run_mx<X128x256<FA>>(g, e, s, st);
        case 5: return run_mx<X128x128<FA>>(g, e, s, st);
        case 6: return run_mx<X128x64<FA>>(g, e, s, st);
        case 7: return run_mx<X64x64<FA>>(g, e, s, st);
        default: break;
    }
    const int nout = e.kind == EP_GATED ? e.F : g.N;
    if (e.kind == EP_GATED) gemm_mx_rows_kernel<FA, 2><<<(nout + 15) / 16, 512, 0, st>>>(g, e, s);
    else gemm_mx_rows_kernel<FA, 1><<<(nout + 15) / 16, 512, 0, st>>>(g, e, s);
    return hipGetLastError();
}

hipError_t launch_gemm_mx(int fmt, const GemmArgs& g, const EpiParams& e, const MxScales& s, int tile, hipStream_t st) {
    if (tile == 0) tile = gemm_mx_tile(fmt, g, e);
    return fmt == MX_FP4 ? run_mx_tile<MX_FP4>(g, e, s, tile, st) : run_mx_tile<MX_FP8>(g, e, s, tile, st);
}

}  // namespace sgd
