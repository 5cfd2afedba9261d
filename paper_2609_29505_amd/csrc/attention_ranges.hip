// Attention in which every query sees an interval of keys: o = sum_j p_j v_j / sum_j p_j over lo <= j < hi,
// p_j = exp(f(q . k_j scale) - slope |pos - j|), f(x) = x or cap tanh(x / cap).  Documents packed into one
// sequence, prefixes, causal order, padding and windows are all such intervals; a query that sees nothing
// gets zeros.  One pass over the keys with a running maximum and sum.  In bf16 the probabilities are rounded to bf16, the
// matrix instruction's operand, for their product with the values; the divisor adds them unrounded in fp32 (8192 packed tokens 2.3e-3 of
// the output against float64, where rounding the output alone gives 1.7e-3).  fp32 rounds nothing below fp32.
//
// Rows of a key head are its queries times the G query heads that share it (row = query G + head), so that
// grouped heads read their keys and values once.  A wave owns 32 rows and computes S^T = K Q^T, as in
// attention.hip: one lane holds one row's scores, and P^T is the right operand of O^T += V^T P^T as it is.  Keys
// and values are read from their token-major rows (any strides): the matrix instruction wants eight keys
// of one dim in a lane, which the transposing LDS read (ds_read_b64_tr_b16) gives from rows stored as they are.
//
// Blocks of 64 keys outside every row's interval are skipped, blocks inside all of a wave's intervals
// are not masked.  A key's value may be infinite or NaN where some rows do not see it (0 x inf is NaN in the
// matrix instruction): blocks that are not wholly visible are looked over for such values, which are
// taken out of the block and added one key at a time to the rows that see them.
//
// Few rows: the keys of a row block are split between workgroups (splits), whose (maximum, sum, O) meet
// in the workspace; in row blocks of 32 the four waves of a workgroup also take different keys.
#include <float.h>

#include <algorithm>

#include "common.h"
#include "gemm_common.h"
#include "kernels.h"
#include "tile_order.h"

namespace sgd {

namespace {
constexpr float kLog2e = 1.44269504088896340736f;
// lazy rescaling: the running maximum is raised only when a block's exceeds it by 2^8 (attention.hip)
constexpr float kSlack = 8.0f;

__device__ __forceinline__ float half_max(float v) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a lane knows of its row
struct Row {
    int lo, hi;      // visible keys; lo = hi: none
    int pos;         // the query's key position, within [lo, hi)
    float slope;     // distance bias, log2 domain
    float c0, c1;    // scores: raw c0 (no cap), or c0 (1 - 2 / (1 + 2^(raw c1)))
};

// The work of a workgroup: a row block and a split of a key head's rows.  Each XCD takes an eighth of the heads
// (tile_order.h), all of them at once, and row blocks from the last to the first: under a causal mask or a prefix
// the long ones start first (8192 causal tokens, 16 heads: 344 us head by head and forwards, 272 so).  Documents of uneven lengths
// come in no such order: nine in 8192 tokens end after 137 block times a place, 106 being the mean.
struct Place { int bh, b, hk, split, rb, G, nr; };
__device__ __forceinline__ Place place_of(const RangeAttnArgs& a, int bx) {
    Place p;
    p.G = a.H / a.Hk;
    p.nr = a.nq * p.G;
    const int per = gridDim.x, heads = gridDim.y, nrb = per / a.splits;
    const int at_once = heads % kXcds ? 1 : heads / kXcds;
    const int pos = tile_position(bx, per * heads);
    const int grp = pos / (at_once * per), rest = pos - grp * (at_once * per), rev = rest / at_once;
    p.bh = grp * at_once + (rest - rev * at_once);
    p.split = (per - 1 - rev) / nrb;
    p.rb = per - 1 - rev - p.split * nrb;
    p.b = p.bh / a.Hk;
    p.hk = p.bh - p.b * a.Hk;
    return p;
}
__device__ __forceinline__ int block_number() { return (int)(blockIdx.y * gridDim.x + blockIdx.x); }
// The kernel's arguments read again, and its block number computed again, through values that the compiler
// cannot see through: the end of a kernel holds no scalars over its main loop
__device__ __forceinline__ const RangeAttnArgs& args_again() {
    const char __attribute__((address_space(4)))* args =
        (const char __attribute__((address_space(4)))*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    return *(const RangeAttnArgs*)(const char*)args;
}
__device__ __forceinline__ int block_again() {
    int n = block_number();
    asm volatile("" : "+s"(n));
    return n;
}

// Query and head of row r of a place's key head (rows past the last: the last one's)
__device__ __forceinline__ void row_place(const Place& p, int r, int& i, int& h) {
    const int rc = min(r, p.nr - 1);
    i = rc / p.G;
    h = p.hk * p.G + (rc - i * p.G);
}
// What its lane knows of it; rows past the last see nothing
template <bool CAP, bool BIAS>
__device__ __forceinline__ Row row_info(const RangeAttnArgs& a, const Place& p, int r, int i, int h) {
    Row w;
    const long at = (long)p.b * a.nq + i;
    w.lo = max(a.ranges[2 * at], 0);
    w.hi = min(a.ranges[2 * at + 1], a.nk);
    if (r >= p.nr || w.lo >= w.hi) w.lo = w.hi = 0;
    // A query outside its interval is moved to the interval's near end: all its distances change by one constant, which
    // the softmax takes out again, and near ones keep fp32's precision (and pos - key its range)
    w.pos = BIAS ? max(min(a.pos ? a.pos[at] : i + a.nk - a.nq, w.hi - 1), w.lo) : 0;
    w.slope = BIAS ? a.slopes[h] * kLog2e : 0.f;
    w.c0 = (CAP ? a.cap : a.scale) * kLog2e;
    w.c1 = CAP ? 2.0f * a.scale * kLog2e / a.cap : 0.f;
    return w;
}

// Union and intersection of the wave's non-empty intervals
struct Span { int lo, hi, ilo, ihi; };
__device__ __forceinline__ Span wave_span(const Row& w) {
    const bool some = w.lo < w.hi;
    Span s{some ? w.lo : INT32_MAX, some ? w.hi : 0, some ? w.lo : 0, some ? w.hi : INT32_MAX};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s.lo = min(s.lo, __shfl_xor(s.lo, o, 64));
        s.hi = max(s.hi, __shfl_xor(s.hi, o, 64));
        s.ilo = max(s.ilo, __shfl_xor(s.ilo, o, 64));
        s.ihi = min(s.ihi, __shfl_xor(s.ihi, o, 64));
    }
    s.lo = __builtin_amdgcn_readfirstlane(s.lo);
    s.hi = __builtin_amdgcn_readfirstlane(s.hi);
    s.ilo = __builtin_amdgcn_readfirstlane(s.ilo);
    s.ihi = __builtin_amdgcn_readfirstlane(s.ihi);
    return s;
}

// Key (relative to the lane's first) of score register r of 32-key group t
__device__ __forceinline__ constexpr int key_of(int t, int r) { return t * 32 + (r >> 2) * 8 + (r & 3); }

// One block's softmax: raw scores s (key of register (t, r): key0 + key_of(t, r)) become probabilities.  The
// running maximum m (log2 domain; -FLT_MAX before the first visible key, so that no difference is NaN) and
// the lane's partial sum go on; returns the factor for what was accumulated before.
// EXACT (fp32 tensors): the cap by tanhf, right to fp32 rounding of small scores too.  Otherwise cap tanh(x / cap) =
// cap - 2 cap R, which is off by 2^-24 cap whatever the score: 2e-6 of a probability at cap 30, where bf16
// probabilities are off by 2e-3.
template <bool CAP, bool BIAS, bool EXACT, int NS>
__device__ __forceinline__ float softmax_block(f32x16 (&s)[NS], const Row& w, int key0, bool masked, float& m, float& lsum) {
    // Without a bias a score's last step, x -> x sf + sb, is folded into the exponent: s holds the raw score (sf = c0,
    // sb = 0) or, capped, R = 1 / (1 + 2^(raw c1)) (sf = -2 c0, sb = c0), and what is masked the value of score -inf
    constexpr bool LATE = !BIAS && !(CAP && EXACT);
    const float sf = LATE ? (CAP ? -2.0f * w.c0 : w.c0) : 1.0f, sb = LATE && CAP ? w.c0 : 0.f;
    const float none = LATE && CAP ? INFINITY : -INFINITY;
    if constexpr (CAP || BIAS) {
        const float d0 = BIAS ? (float)(w.pos - key0) : 0.f;
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float x = s[t][r];
                if constexpr (CAP && EXACT) {
                    x = w.c0 * tanhf(x * (w.c1 * 0.5f / kLog2e));
                } else if constexpr (CAP) {
                    x = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * w.c1));
                    if constexpr (BIAS) x = fmaf(-2.0f * w.c0, x, w.c0);
                } else {
                    x *= w.c0;
                }
                if constexpr (BIAS) x = fmaf(-w.slope, fabsf(d0 - (float)key_of(t, r)), x);
                s[t][r] = x;
            }
    }
    if (masked) {
        const unsigned a = (unsigned)(w.lo - key0), n = (unsigned)(w.hi - w.lo);
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if ((unsigned)key_of(t, r) - a >= n) s[t][r] = none;
                if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // a few conditions at a time: they take scalars
            }
    }
    constexpr float sign = LATE && CAP ? -1.0f : 1.0f;  // the largest score has the smallest R
    float bm = -INFINITY;
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) bm = fmaxf(bm, sign * s[t][r]);
    bm = half_max(bm);
    if constexpr (LATE) bm = fmaf(sign * bm, sf, sb);
    float alpha = 1.0f;
    if (__builtin_amdgcn_ballot_w64(bm > m + kSlack)) {
        const float mn = fmaxf(m, bm);
        alpha = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        lsum *= alpha;
    }
    const float at = sb - m;
    float ps = 0.f;
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = __builtin_amdgcn_exp2f(LATE ? fmaf(s[t][r], sf, at) : s[t][r] - m);
            s[t][r] = p;
            ps += p;
        }
    lsum += ps;
    return alpha;
}

// Where a row's partial result goes: [split][b Hk + hk][row][dh + 4] fp32: O, then the maximum and the sum
__device__ __forceinline__ float* partial_row(const RangeAttnArgs& a, int split, int bh, int r) {
    const long nr = (long)a.nq * (a.H / a.Hk);
    return (float*)a.work + (((long)split * a.B * a.Hk + bh) * nr + r) * (a.dh + 4);
}

// A lane's O^T (dims dt 32 + 8 (r / 4) + 4 half + r % 4 of its row), maximum and whole sum: divided and
// stored, or left for the join.  A wave's bf16 rows go through LDS (stage: 32 rows of DT 64 + 16 bytes of the wave's
// own): straight from the registers a store would touch 16 bytes of each of 32 rows.
template <int DT, typename T, int RPB>
__device__ __forceinline__ void finish(const f32x16 (&o)[DT], const Row& w, float m, float l, int wave_row, int lane, char* stage) {
    const RangeAttnArgs& a = args_again();
    const Place pl = place_of(a, block_again());
    const int half = lane >> 5, r0 = pl.rb * RPB + wave_row, r = r0 + (lane & 31);
    const bool some = w.lo < w.hi;
    const float inv = 1.0f / l;
    int dh = a.dh;
    if (a.splits > 1 || sizeof(T) == 4) {
        if (r >= pl.nr) return;
        int i, h;
        row_place(pl, r, i, h);
        float* const dst = a.splits > 1 ? partial_row(a, pl.split, pl.bh, r) : (float*)a.o + pl.b * a.os[0] + i * a.os[1] + h * a.os[2];
        const float f = a.splits > 1 ? 1.f : some ? inv : 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                asm volatile("" : "+s"(dh));  // one condition at a time
                if (dt * 32 + g * 8 >= dh) continue;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = a.splits > 1 || some ? o[dt][4 * g + e] * f : 0.f;
                *(f32x4*)(dst + dt * 32 + g * 8 + half * 4) = v;
            }
        if (a.splits > 1 && half == 0) {
            dst[dh] = m;
            dst[dh + 1] = some ? l : -1.0f;  // -1: the row sees nothing
        }
        return;
    }
    if constexpr (sizeof(T) == 2) {
        constexpr int P = DT * 64 + 16;  // bytes of a staged row
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = some ? o[dt][4 * g + e] * inv : 0.f;
                store_bf16x4((bf16*)(stage + (lane & 31) * P) + dt * 32 + g * 8 + half * 4, v);
            }
        asm volatile("" ::: "memory");  // the reads stay behind the writes (a wave's LDS operations are in order)
        const int per = dh / 8;  // 16-byte pieces of a row
        for (int x = lane; x < 32 * per; x += 64) {
            const int row = x / per, c = x - row * per;
            if (r0 + row >= pl.nr) break;
            int i, h;
            row_place(pl, r0 + row, i, h);
            const u32x4 v = *(const u32x4*)(stage + row * P + c * 16);
            bf16* const dst = (bf16*)a.o + pl.b * a.os[0] + i * a.os[1] + h * a.os[2] + c * 8;
            *(u32x2*)dst = u32x2{v[0], v[1]};
            *(u32x2*)(dst + 4) = u32x2{v[2], v[3]};
        }
    }
}

// Bits of a pair of bf16 values: 0x8000 in each half that holds an infinity or a NaN
__device__ __forceinline__ uint32_t odd_pair(uint32_t x) { return ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }

// Looks over 16 bytes of values in LDS and clears infinities and NaN there; whether there were any
__device__ __forceinline__ bool clear_odd(char* p) {
    u32x4 x = *(const u32x4*)p;
    uint32_t odd = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= odd_pair(x[e]);
    if (odd) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] &= ~((odd_pair(x[e]) >> 15) * 0xFFFFu);
        *(u32x4*)p = x;
    }
    return odd != 0;
}

// The infinities and NaN that were cleared from a block, added to the rows that see them: keys [j0, j1), read
// again from memory one at a time (V: key 0, ts elements a key)
template <int DT, typename T>
__device__ __forceinline__ void add_odd(f32x16 (&o)[DT], const Row& w, const T* V, long ts, int j0, int j1, int dh, int half) {
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
        const bool see = j >= w.lo && j < w.hi;
        const T* const p = V + j * ts + half * 4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                asm volatile("" : "+s"(dh));  // sixteen addresses kept over the main loop would spill
                const int d = min(dt * 32 + g * 8, dh - 8);  // what lies past dh is not stored
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = ElemIO<T>::load(p + d + e);
                    o[dt][4 * g + e] += see && !(fabsf(v) <= FLT_MAX) ? v : 0.f;
                }
                __builtin_amdgcn_sched_barrier(0);  // a rare path: it takes no registers from the others
            }
    }
}

// K and V tiles in LDS, bf16: rows of P bytes, 16-byte chunks swizzled
template <int DH> struct Tile {
    static constexpr int P = DH <= 64 ? 128 : 256, CH = P / 16;
    static constexpr int KS = DH / 16, DT = DH / 32;
    // fragment reads of 16 consecutive keys cover the 64 banks once
    __device__ static __forceinline__ int kpos(int key, int c) { return P == 256 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); }
    // a transposing read takes 64 bytes of each of four consecutive keys: in different banks
    __device__ static __forceinline__ int vpos(int key, int c) { return P == 256 ? c ^ ((key & 3) << 2) : c ^ (((key >> 1) & 1) << 2); }
};

typedef __bf16 __attribute__((ext_vector_type(4))) tr4;
__device__ __forceinline__ bf16x4 read_tr(const char* p) {
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((tr4 __attribute__((address_space(3)))*)(__attribute__((address_space(3))) char*)p));
}

// V^T fragment of 16-key group k16 (keys 16 k16 + 4 half + 0..3 and + 8), dims 32 dt + lane % 32; at: the lane's
// place in its tile for group 0, dims 0
template <int DH>
struct VRead {
    const char* p[Tile<DH>::DT];
    __device__ __forceinline__ VRead(const char* tile, int lane) {
        const int half = lane >> 5, i = lane & 15, key = half * 4 + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < Tile<DH>::DT; ++dt) {
            const int d = dt * 32 + ((lane >> 4) & 1) * 16 + (i & 3) * 4;
            p[dt] = tile + key * Tile<DH>::P + Tile<DH>::vpos(key, d >> 3) * 16 + (d & 4) * 2;
        }
    }
    // the swizzle depends on the key's last two bits only: steps of eight keys keep it
    __device__ __forceinline__ bf16x8 frag(int off, int dt, int k16) const {
        const bf16x4 a = read_tr(p[dt] + off + k16 * 16 * Tile<DH>::P), b = read_tr(p[dt] + off + (k16 * 16 + 8) * Tile<DH>::P);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// O^T += V^T P^T over NS x 32 keys
template <int DH, int NS>
__device__ __forceinline__ void pv_block(const VRead<DH>& v, int off, const f32x16 (&s)[NS], f32x16 (&o)[Tile<DH>::DT]) {
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
            bf16x8 pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[e] = f2bf(s[t][8 * k2 + e]);
#pragma unroll
            for (int dt = 0; dt < Tile<DH>::DT; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.frag(off, dt, t * 2 + k2), pf, o[dt], 0, 0, 0);
        }
}

// the part of [first, last) (blocks) that split s of n takes
__device__ __forceinline__ void split_blocks(int& first, int& last, int s, int n) {
    const int c = (last - first + n - 1) / n;
    first = min(first + s * c, last);
    last = min(first + c, last);
}

// the lane's query row as right operand: dims 16 ks + 8 half .. + 7 (zeros from dh on)
template <int KS>
__device__ __forceinline__ void load_q(bf16x8 (&q)[KS], const bf16* p, int dh, int half) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int c = ks * 16 + half * 8;
        bf16x8 z;
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = f2bf(0.f);
        q[ks] = c < dh ? *(const bf16x8*)(p + c) : z;
    }
}

// The results of a workgroup's NW waves for the same rows, joined in wave 0 in their order (mg: wave_bytes a wave); returns
// the common maximum
template <int DT> constexpr int wave_bytes = (DT * 16 + 2) * 64 * 4;
template <int DT, int NW>
__device__ __forceinline__ float join_waves(f32x16 (&o)[DT], float m, float& lsum, float* mg, int wave, int lane) {
    constexpr int ST = wave_bytes<DT> / 4;
    __syncthreads();  // the blocks' LDS is free
    if (wave) {
        float* const p = mg + wave * ST + lane;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) p[(t * 16 + e) * 64] = o[t][e];
        p[DT * 16 * 64] = m;
        p[(DT * 16 + 1) * 64] = lsum;
    }
    __syncthreads();
    if (wave) return m;
    float mx = m;
#pragma unroll
    for (int k = 1; k < NW; ++k) mx = fmaxf(mx, mg[k * ST + DT * 16 * 64 + lane]);
    {
        const float f = __builtin_amdgcn_exp2f(m - mx);
        lsum *= f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[t][e] *= f;
    }
#pragma unroll
    for (int k = 1; k < NW; ++k) {
        const float* const p = mg + k * ST + lane;
        const float f = __builtin_amdgcn_exp2f(p[DT * 16 * 64] - mx);
        lsum = fmaf(p[(DT * 16 + 1) * 64], f, lsum);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[t][e] = fmaf(p[(t * 16 + e) * 64], f, o[t][e]);
    }
    return mx;
}
}  // namespace

// --------------------------------------------------------------------------- bf16, many rows
//
// Four waves, 128 rows, blocks of 64 keys double-buffered in LDS (64 KB at 128 dims: two workgroups a
// CU, one's vector instructions under the other's matrix instructions).  The next block's loads are issued after the
// barrier that opens a block and waited for at the next one.

template <int DH, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void range_attn_bf16_kernel(RangeAttnArgs a) {
    using T = Tile<DH>;
    constexpr int BKV = 64, NW = 4, NT = NW * 64, TB = BKV * T::P, LP = TB / (NT * 16), RP = NT / T::CH;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TB];  // K, V of buffer 0, then of buffer 1
    __shared__ int wspan[NW][4];
    __shared__ int odd_at[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const Place pl = place_of(a, block_number());
    const int r = pl.rb * 128 + wave * 32 + (lane & 31);
    int i, h;
    row_place(pl, r, i, h);
    bf16x8 qf[T::KS];
    load_q(qf, (const bf16*)a.q + pl.b * a.qs[0] + i * a.qs[1] + h * a.qs[2], a.dh, half);
    const Row w = row_info<CAP, BIAS>(a, pl, r, i, h);
    const Span ws = wave_span(w);
    if (lane == 0) { wspan[wave][0] = ws.lo; wspan[wave][1] = ws.hi; wspan[wave][2] = ws.ilo; wspan[wave][3] = ws.ihi; }
    if (tid < 2) odd_at[tid] = -1;
    __syncthreads();
    Span gs = ws;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
        gs.lo = min(gs.lo, wspan[k][0]);
        gs.hi = max(gs.hi, wspan[k][1]);
    }
    gs.lo = __builtin_amdgcn_readfirstlane(gs.lo);
    gs.hi = __builtin_amdgcn_readfirstlane(gs.hi);
    // lane w < 4 holds wave w's span
    const int sl = lane < NW ? lane : 0;
    const Span of_wave{lane < NW ? wspan[sl][0] : INT32_MAX, lane < NW ? wspan[sl][1] : 0, wspan[sl][2], wspan[sl][3]};
    int first = 0, last = 0;
    if (gs.lo < gs.hi) {
        first = gs.lo / BKV;
        last = (gs.hi + BKV - 1) / BKV;
    }
    split_blocks(first, last, pl.split, a.splits);

    const bf16* const K = (const bf16*)a.k + pl.b * a.ks[0] + pl.hk * a.ks[2];
    const bf16* const V = (const bf16*)a.v + pl.b * a.vs[0] + pl.hk * a.vs[2];
    // load part p: rows p RP + tid / CH, LDS chunk tid % CH
    const int prow = tid / T::CH, pch = tid % T::CH;
    unsigned ko[LP], vo[LP];
#pragma unroll
    for (int p = 0; p < LP; ++p) {
        const int row = p * RP + prow, ck = T::kpos(row, pch), cv = T::vpos(row, pch);
        ko[p] = ck * 8 < a.dh ? (unsigned)(row * a.ks[1] * 2 + ck * 16) : 0xFFFFFF00u;
        vo[p] = cv * 8 < a.dh ? (unsigned)(row * a.vs[1] * 2 + cv * 16) : 0xFFFFFF00u;
    }
    const unsigned l0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * 1024;
    auto load = [&](int kb, int buf) {
        asm volatile("" : "+s"(kb));  // the addresses are computed here, not carried through the loop
        const long k0 = (long)kb * BKV;
        const unsigned rows = (unsigned)min((long)BKV, a.nk - k0) - 1;
        const u32x4 rk = buf_desc(K + k0 * a.ks[1], rows * (unsigned)(a.ks[1] * 2) + a.dh * 2);
        const u32x4 rv = buf_desc(V + k0 * a.vs[1], rows * (unsigned)(a.vs[1] * 2) + a.dh * 2);
#pragma unroll
        for (int p = 0; p < LP; ++p) dma16(l0 + buf * 2 * TB + p * NT * 16, ko[p], rk, 0);
#pragma unroll
        for (int p = 0; p < LP; ++p) dma16(l0 + buf * 2 * TB + TB + p * NT * 16, vo[p], rv, 0);
    };
    const char* kf[T::KS];
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) kf[ks] = lds + (lane & 31) * T::P + T::kpos(lane & 31, ks * 2 + half) * 16;
    const VRead<DH> vf(lds + TB, lane);

    f32x16 o[T::DT];
#pragma unroll
    for (int t = 0; t < T::DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
    float m = -FLT_MAX, lsum = 0.f;
    if (first < last) load(first, 0);
    // the query rows are here: left open, the compiler would wait for them, and with them for the next
    // block's loads, before the first matrix instruction of every block
    __builtin_amdgcn_s_waitcnt(0);
    for (int kb = first; kb < last; ++kb) {
        const int k0 = kb * BKV, buf = (kb - first) & 1, off = buf * 2 * TB;
        // whether some wave sees only a part of it (a wave that sees nothing of it passes it over)
        const bool part = __builtin_amdgcn_ballot_w64(k0 < of_wave.hi && k0 + BKV > of_wave.lo && (k0 < of_wave.ilo || k0 + BKV > of_wave.ihi));
        vm_wait<0>();
        if (part) {  // each thread looks over the values that it brought
            bool odd = false;
#pragma unroll
            for (int p = 0; p < LP; ++p) odd |= clear_odd(lds + off + TB + p * NT * 16 + tid * 16);
            if (odd) odd_at[buf] = kb;
        }
        __syncthreads();
        if (kb + 1 < last) load(kb + 1, buf ^ 1);
        if (k0 >= ws.hi || k0 + BKV <= ws.lo) continue;
        f32x16 s[2];
        // Wide heads: all of K's fragments are read first, then half of V's between the scores' instructions (4096
        // tokens, 32 heads of 128 dims: 273 us, left to the compiler 288; of 64 dims 169 either way)
        constexpr bool AHEAD = DH > 64;
        constexpr int NK = 2 * T::KS, NV = 4 * T::DT, NP = AHEAD ? NV / 2 : 0;
        bf16x8 kr[AHEAD ? NK : 1], vr[AHEAD ? NP : 1];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
        if constexpr (AHEAD) {
#pragma unroll
            for (int x = 0; x < NK; ++x) kr[x] = *(const bf16x8*)(kf[x >> 1] + off + (x & 1) * 32 * T::P);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < NK; ++x) {
                s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr[x], qf[x >> 1], s[x & 1], 0, 0, 0);
#pragma unroll
                for (int y = x * NP / NK; y < (x + 1) * NP / NK; ++y) vr[y] = vf.frag(off, y % T::DT, y / T::DT);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ks = 0; ks < T::KS; ++ks)
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kf[ks] + off + t * 32 * T::P), qf[ks], s[t], 0, 0, 0);
        }
        const bool masked = k0 < ws.ilo || k0 + BKV > ws.ihi;
        const float alpha = softmax_block<CAP, BIAS, false, 2>(s, w, k0 + half * 4, masked, m, lsum);
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f))
#pragma unroll
            for (int t = 0; t < T::DT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            bf16x8 pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[e] = f2bf(s[k >> 1][8 * (k & 1) + e]);
#pragma unroll
            for (int dt = 0; dt < T::DT; ++dt) {
                const int y = k * T::DT + dt;
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y < NP ? vr[y < NP ? y : 0] : vf.frag(off, dt, k), pf, o[dt], 0, 0, 0);
            }
        }
        if (part && __builtin_amdgcn_readfirstlane(odd_at[buf]) == kb)
            add_odd<T::DT, bf16>(o, w, V, a.vs[1], max(k0, ws.lo), min(k0 + BKV, ws.hi), a.dh, half);
    }
    __syncthreads();  // the blocks' LDS is free
    finish<T::DT, bf16, 128>(o, w, m, half_sum(lsum), wave * 32, lane, lds + wave * 32 * (T::DT * 64 + 16));
}

// --------------------------------------------------------------------------- bf16, 32 rows a workgroup
//
// For single tokens the keys are read once and the kernel is bound by memory; for short prompts it is there to fill the
// chip.  Each of four waves takes every fourth 32-key block of the workgroup's split, with two blocks of its own in LDS
// (32 KB a wave at 128 dims) and no barrier until the waves' results are joined (8 sequences of up to 16384 keys, 8 key heads, 416 MB: 90 us with the join, 4.6 TB/s).

template <int DH, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 1) void range_attn_few_kernel(RangeAttnArgs a) {
    using T = Tile<DH>;
    constexpr int BKV = 32, NW = 4, TB = BKV * T::P, LP = TB / 1024, RP = 64 / T::CH;
    constexpr int BYTES = NW * std::max(4 * TB, wave_bytes<T::DT>);
    __shared__ __attribute__((aligned(1024))) char lds[BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const Place pl = place_of(a, block_number());
    const int r = pl.rb * 32 + (lane & 31);
    int i, h;
    row_place(pl, r, i, h);
    bf16x8 qf[T::KS];
    load_q(qf, (const bf16*)a.q + pl.b * a.qs[0] + i * a.qs[1] + h * a.qs[2], a.dh, half);
    const Row w = row_info<CAP, BIAS>(a, pl, r, i, h);
    const Span ws = wave_span(w);
    int first = 0, last = 0;
    if (ws.lo < ws.hi) {
        first = ws.lo / BKV;
        last = (ws.hi + BKV - 1) / BKV;
    }
    split_blocks(first, last, pl.split, a.splits);

    const bf16* const K = (const bf16*)a.k + pl.b * a.ks[0] + pl.hk * a.ks[2];
    const bf16* const V = (const bf16*)a.v + pl.b * a.vs[0] + pl.hk * a.vs[2];
    const int prow = lane / T::CH, pch = lane % T::CH;
    unsigned ko[LP], vo[LP];
#pragma unroll
    for (int p = 0; p < LP; ++p) {
        const int row = p * RP + prow, ck = T::kpos(row, pch), cv = T::vpos(row, pch);
        ko[p] = ck * 8 < a.dh ? (unsigned)(row * a.ks[1] * 2 + ck * 16) : 0xFFFFFF00u;
        vo[p] = cv * 8 < a.dh ? (unsigned)(row * a.vs[1] * 2 + cv * 16) : 0xFFFFFF00u;
    }
    char* const mine = lds + wave * 4 * TB;  // K, V of buffer 0, then of buffer 1
    const unsigned l0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * 4 * TB;
    // block kb into a buffer; nothing but zeros past the last (the counted waits need every load)
    auto load = [&](int kb, int buf) {
        const bool in = kb < last;
        const long k0 = in ? (long)kb * BKV : 0;
        const unsigned rows = (unsigned)min((long)BKV, a.nk - k0) - 1;
        const u32x4 rk = buf_desc(K + k0 * a.ks[1], in ? rows * (unsigned)(a.ks[1] * 2) + a.dh * 2 : 0);
        const u32x4 rv = buf_desc(V + k0 * a.vs[1], in ? rows * (unsigned)(a.vs[1] * 2) + a.dh * 2 : 0);
#pragma unroll
        for (int p = 0; p < LP; ++p) dma16(l0 + buf * 2 * TB + p * 1024, ko[p], rk, 0);
#pragma unroll
        for (int p = 0; p < LP; ++p) dma16(l0 + buf * 2 * TB + TB + p * 1024, vo[p], rv, 0);
    };
    const char* kf[T::KS];
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) kf[ks] = mine + (lane & 31) * T::P + T::kpos(lane & 31, ks * 2 + half) * 16;
    const VRead<DH> vf(mine + TB, lane);
    f32x16 o[T::DT];
#pragma unroll
    for (int t = 0; t < T::DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
    float m = -FLT_MAX, lsum = 0.f;
    __builtin_amdgcn_s_waitcnt(0);  // the query rows are here (as above; not after the two loads, whose wait is counted)
    load(first + wave, 0);
    load(first + wave + NW, 1);
    int buf = 0;
    for (int kb = first + wave; kb < last; kb += NW, buf ^= 1) {
        const int k0 = kb * BKV, off = buf * 2 * TB;
        vm_wait<2 * LP>();
        const bool masked = k0 < ws.ilo || k0 + BKV > ws.ihi;
        bool odd = false;
        if (masked) {
#pragma unroll
            for (int p = 0; p < LP; ++p) odd |= clear_odd(mine + off + TB + p * 1024 + lane * 16);
        }
        f32x16 s[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks)
            s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kf[ks] + off), qf[ks], s[0], 0, 0, 0);
        const float alpha = softmax_block<CAP, BIAS, false, 1>(s, w, k0 + half * 4, masked, m, lsum);
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f))
#pragma unroll
            for (int t = 0; t < T::DT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
        pv_block<DH, 1>(vf, off, s, o);
        if (masked && __builtin_amdgcn_ballot_w64(odd))
            add_odd<T::DT, bf16>(o, w, V, a.vs[1], max(k0, ws.lo), min(k0 + BKV, ws.hi), a.dh, half);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the buffer has been read
        load(kb + 2 * NW, buf);
    }
    vm_wait<0>();
    m = join_waves<T::DT, NW>(o, m, lsum, (float*)lds, wave, lane);
    if (wave) return;
    finish<T::DT, bf16, 32>(o, w, m, half_sum(lsum), 0, lane, lds);
}

// --------------------------------------------------------------------------- fp32
//
// The same with fp32 matrix instructions (32x32x2: a lane's left operand is one value): dims are taken in the
// order 8 j + 4 half + 0..3, so that a lane reads four at once, and values as they lie in their
// rows.  Blocks of 32 keys come through registers, the next one's loads under this one's instructions (4096 tokens, 8
// heads of 128 dims 647 us, 106 TFLOP/s of the 154 that a large product reaches; loaded when needed 835).
// FEW: 32 rows a workgroup, which all four waves hold, each with every fourth block in LDS of its own and no barrier
// before the join (one token, 16384 keys, 32 heads 125 us, 4.3 TB/s; in one wave of the other form 462); otherwise four waves
// of 32 rows share a block.

template <int DH, bool CAP, bool BIAS, bool FEW>
__global__ __launch_bounds__(256, 1) void range_attn_f32_kernel(RangeAttnArgs a) {
    constexpr int BKV = 32, NW = 4, DT = DH / 32, J = DH / 8, P = DH + 4;  // padded rows
    constexpr int NL = FEW ? 64 : 256, C4 = DH / 4, PER = BKV * C4 / NL;   // threads that bring a block, each PER pieces of K and V
    constexpr int BLOCK = 2 * BKV * P, FLOATS = FEW ? NW * std::max(BLOCK, wave_bytes<DT> / 4) : BLOCK;
    __shared__ __attribute__((aligned(16))) float lds[FLOATS];
    __shared__ int wspan[NW][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const Place pl = place_of(a, block_number());
    const int r = FEW ? pl.rb * 32 + l32 : pl.rb * 128 + wave * 32 + l32;
    int i, h;
    row_place(pl, r, i, h);
    const Row w = row_info<CAP, BIAS>(a, pl, r, i, h);
    const Span ws = wave_span(w);
    int lo = ws.lo, hi = ws.hi, first = 0, last = 0;
    if constexpr (!FEW) {
        if (lane == 0) { wspan[wave][0] = ws.lo; wspan[wave][1] = ws.hi; }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NW; ++k) { lo = min(lo, wspan[k][0]); hi = max(hi, wspan[k][1]); }
    }
    if (lo < hi) { first = lo / BKV; last = (hi + BKV - 1) / BKV; }
    split_blocks(first, last, pl.split, a.splits);
    const float* const Q = (const float*)a.q + pl.b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
    const float* const K = (const float*)a.k + pl.b * a.ks[0] + pl.hk * a.ks[2];
    const float* const V = (const float*)a.v + pl.b * a.vs[0] + pl.hk * a.vs[2];
    float* const sk = lds + (FEW ? wave * BLOCK : 0);
    float* const sv = sk + BKV * P;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 qf[J];
#pragma unroll
    for (int j = 0; j < J; ++j) qf[j] = 8 * j + 4 * half < a.dh ? *(const f32x4*)(Q + 8 * j + 4 * half) : zero;
    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
    float m = -FLT_MAX, lsum = 0.f;
    f32x4 kr[PER], vr[PER];
    const int me = FEW ? lane : tid;
    auto fetch = [&](int kb) {
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int x = p * NL + me, row = x / C4, c = (x - row * C4) * 4;
            const long key = (long)kb * BKV + row;
            const bool in = key < a.nk && c < a.dh;
            kr[p] = in ? *(const f32x4*)(K + key * a.ks[1] + c) : zero;
            vr[p] = in ? *(const f32x4*)(V + key * a.vs[1] + c) : zero;
        }
    };
    const int step = FEW ? NW : 1;
    int kb = first + (FEW ? wave : 0);
    if (kb < last) fetch(kb);
    for (; kb < last; kb += step) {
        const int k0 = kb * BKV;
        bool odd = false;
        if constexpr (!FEW) __syncthreads();  // the last block has been read
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int x = p * NL + me, row = x / C4, c = (x - row * C4) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(fabsf(vr[p][e]) <= FLT_MAX)) { odd = true; vr[p][e] = 0.f; }
            *(f32x4*)(sk + row * P + c) = kr[p];
            *(f32x4*)(sv + row * P + c) = vr[p];
        }
        if constexpr (FEW) {
            odd = __builtin_amdgcn_ballot_w64(odd) != 0;
            asm volatile("" ::: "memory");  // a wave's LDS operations are in order
        } else {
            odd = __builtin_amdgcn_readfirstlane(__syncthreads_or(odd));
        }
        if (kb + step < last) fetch(kb + step);
        if (k0 >= ws.hi || k0 + BKV <= ws.lo) continue;
        f32x16 s[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const f32x4 kf = *(const f32x4*)(sk + l32 * P + 8 * j + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[j][e], s[0], 0, 0, 0);
        }
        const bool masked = k0 < ws.ilo || k0 + BKV > ws.ihi;
        const float alpha = softmax_block<CAP, BIAS, true, 1>(s, w, k0 + half * 4, masked, m, lsum);
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f))
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
        const float* const vl = sv + half * 4 * P + l32;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(vl[key_of(0, e) * P + t * 32], s[0][e], o[t], 0, 0, 0);
        if (odd) add_odd<DT, float>(o, w, V, a.vs[1], max(k0, ws.lo), min(k0 + BKV, ws.hi), a.dh, half);
        if constexpr (FEW) asm volatile("" ::: "memory");  // before the next block is written
    }
    if constexpr (FEW) {
        m = join_waves<DT, NW>(o, m, lsum, lds, wave, lane);
        if (wave) return;
    }
    finish<DT, float, FEW ? 32 : 128>(o, w, m, half_sum(lsum), FEW ? 0 : wave * 32, lane, nullptr);
}

// --------------------------------------------------------------------------- join of splits
//
// O = sum_s O_s 2^(m_s - m) / sum_s l_s 2^(m_s - m), four dims a lane; lane s holds split s's maximum and factor.  Few rows:
// the eight half waves of a workgroup take every eighth split of one row (FEW false); many rows: half a wave a row (512 query
// rows of 32 heads, 2 splits: the whole call 29 us, a workgroup a row 43; 100 rows of 8 heads, 16 splits 18.4 and 14.9; a
// token of 32 heads, 8 splits 53 and 50).
template <typename T, bool FEW>
__global__ __launch_bounds__(256) void range_attn_join_kernel(RangeAttnArgs a) {
    constexpr int PARTS = FEW ? 1 : 8, W = FEW ? 32 : 64;  // half waves of a row, lanes that know its splits
    __shared__ f32x4 part[8][32];
    const int l32 = threadIdx.x & 31, hw = threadIdx.x >> 5, c = l32 * 4;
    const long G = a.H / a.Hk, nr = a.nq * G, rows = (long)a.B * a.Hk * nr, at = FEW ? blockIdx.x * 8L + hw : blockIdx.x;  // over [bh][r]
    const long row = min(at, rows - 1), stride = rows * (a.dh + 4);
    const float* const p = (const float*)a.work + row * (a.dh + 4);
    const int mine = FEW ? l32 : threadIdx.x & 63;  // this lane's split
    const float m = mine < a.splits ? p[mine * stride + a.dh] : -FLT_MAX;
    const float l = mine < a.splits ? p[mine * stride + a.dh + 1] : 0.f;
    float mx = m, none = l;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
        mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        none = fminf(none, __shfl_xor(none, o, 64));
    }
    const float factor = __builtin_amdgcn_exp2f(m - mx);
    float sum = l * factor;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < a.splits; s0 += PARTS) {
        const int s = FEW ? s0 : s0 + hw;
        const float f = __shfl(factor, s & (W - 1), W);
        if (s < a.splits && c < a.dh) o += *(const f32x4*)(p + s * stride + c) * f;
    }
    if constexpr (!FEW) {
        part[hw][l32] = o;
        __syncthreads();
        if (hw) return;
#pragma unroll
        for (int k = 1; k < 8; ++k) o += part[k][l32];
    }
    if (at >= rows || c >= a.dh) return;
    const bool some = !(none < 0.f);
    const float inv = 1.0f / sum;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = some ? o[e] * inv : 0.f;
    const long bh = row / nr, r = row - bh * nr;
    const long b = bh / a.Hk, hk = bh - b * a.Hk, i = r / G, h = hk * G + (r - i * G);
    T* const dst = (T*)a.o + b * a.os[0] + i * a.os[1] + h * a.os[2] + c;
    if constexpr (sizeof(T) == 2) store_bf16x4((bf16*)dst, v);
    else *(f32x4*)dst = f32x4{v[0], v[1], v[2], v[3]};
}

// --------------------------------------------------------------------------- dispatch

// Rows of a workgroup: 32, which its waves share with different keys, or 128, a wave's 32 each.  Past 32 rows a key head
// the first is for calls whose 128-row blocks leave CUs empty: its workgroups have to fit one round (one a CU, two up to
// 64 dims), and, as four times as many read every key, have few keys.  us in blocks of 32 and 128 rows, 32 heads: 64 dims,
// bf16, 333 rows and keys 11.0 and 11.7, 512 rows and 1024 keys 16.4 and 23.0, 128 rows and 8192 keys 37.4 and 29.6; fp32,
// 128 rows and 333 keys 16.7 and 26.5, 512 rows and 2048 keys 117 and 104; 128 dims, bf16, 200 rows and 1024 keys 20.0 and
// 22.9, and 2048 keys 28.5 and 26.0, 8 heads of 64 rows and 512 keys 13.2 and 11.4; fp32, 200 rows and 333 keys 27.4 and
// 43.4, 128 rows and 2048 keys 65 and 60.
static int block_rows(int bf, const RangeAttnArgs& a) {
    const long nr = (long)a.nq * (a.H / a.Hk), groups = (nr + 31) / 32 * a.B * a.Hk, reads = groups * a.nk;
    if (nr <= 32) return 32;
    if (a.dh <= 64) return groups <= 512 && (reads <= 1L << 19 || (bf && groups > 256)) ? 32 : 128;
    return groups <= 256 && reads < 1L << 18 && (!bf || (groups > 64 && a.nk >= 256)) ? 32 : 128;
}
static long row_blocks(int bf, const RangeAttnArgs& a) {
    const long nr = (long)a.nq * (a.H / a.Hk), rows = block_rows(bf, a);
    return (nr + rows - 1) / rows;
}

// Splits that give every CU one workgroup and each of them at least 128 keys (the kernel for few rows has one
// workgroup a CU: 16384 keys, 32 key heads, 8 splits 70 us, 16 in two rounds 77, 32 92; 1024 keys, 8 key heads, bf16: 8 splits
// 12.1 us, 4 13.2, whole 16.6; 600 keys, 32 key heads, fp32: 4 splits 22.4, whole 38.0).  In bf16 two splits of fewer than 1024
// keys do not pay for their join (512 keys, 128 key heads 16.7 us, whole 13.9).
int range_attention_splits(int bf, const RangeAttnArgs& a) {
    const long groups = a.B * a.Hk * row_blocks(bf, a);
    const long n = std::min({256L / groups, a.nk / 128L, 64L});
    return n <= 1 || (bf && n == 2 && a.nk < 1024) ? 1 : (int)n;
}

size_t range_attention_bytes(const RangeAttnArgs& a, int splits) {
    return splits <= 1 ? 0 : (size_t)splits * a.B * a.H * a.nq * (a.dh + 4) * sizeof(float);
}

template <int DH, bool CAP, bool BIAS>
static void range_run(int bf, const RangeAttnArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(row_blocks(bf, a) * a.splits), (unsigned)(a.B * a.Hk));
    const bool few = block_rows(bf, a) == 32;
    if (!bf) few ? range_attn_f32_kernel<DH, CAP, BIAS, true><<<grid, 256, 0, st>>>(a)
                 : range_attn_f32_kernel<DH, CAP, BIAS, false><<<grid, 256, 0, st>>>(a);
    else if (few) range_attn_few_kernel<DH, CAP, BIAS><<<grid, 256, 0, st>>>(a);
    else range_attn_bf16_kernel<DH, CAP, BIAS><<<grid, 256, 0, st>>>(a);
}
template <int DH>
static void range_modes(int bf, const RangeAttnArgs& a, hipStream_t st) {
    if (a.cap > 0.f) a.slopes ? range_run<DH, true, true>(bf, a, st) : range_run<DH, true, false>(bf, a, st);
    else a.slopes ? range_run<DH, false, true>(bf, a, st) : range_run<DH, false, false>(bf, a, st);
}

hipError_t launch_range_attention(int bf, const RangeAttnArgs& a, hipStream_t st) {
    if (a.dh <= 64) range_modes<64>(bf, a, st);
    else if (a.dh <= 96) range_modes<96>(bf, a, st);
    else range_modes<128>(bf, a, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits <= 1) return e;
    const long rows = (long)a.B * a.H * a.nq;
    if (a.splits <= 16 && rows >= 4096) {
        const dim3 grid((unsigned)((rows + 7) / 8));
        if (bf) range_attn_join_kernel<bf16, true><<<grid, 256, 0, st>>>(a);
        else range_attn_join_kernel<float, true><<<grid, 256, 0, st>>>(a);
    } else {
        if (bf) range_attn_join_kernel<bf16, false><<<dim3((unsigned)rows), 256, 0, st>>>(a);
        else range_attn_join_kernel<float, false><<<dim3((unsigned)rows), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace sgd
