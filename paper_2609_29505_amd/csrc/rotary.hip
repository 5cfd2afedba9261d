// Rotation of head dims by their token's position (rotary positions).
//
// Pair p of a head turns by the angle 2 pi pos turns[p]: (u, w) -> (u cos - w sin, w cos + u sin), where
// (u, w) are dims p and p + rot / 2 (half layout) or 2 p and 2 p + 1 (interleaved).  Dims from rot on are
// copied.  The turn count is a product in fp64, of which only the fraction goes on (v_sin_f32 and
// v_cos_f32 take turns): at position 10^6 an fp32 count would be off by a sixteenth of a turn.  The fraction and the
// instructions are fp32: fp32 results are off by 2^-22.3 of the sum of a pair's magnitudes at most, 7e-8 rms (with sines rounded once
// from fp64 2^-22.9, 4e-8), at any position.
//
// Bound by memory: every value is read and written once.  A thread takes V neighbouring values of u and of w
// (V = 8 16-bit values: 16 bytes) for one token, computes their angles once and applies them to
// every hl_n-th head of a workgroup, so that the sines cost a fraction of the traffic's time (16384 tokens, 64 heads of 128
// bf16 dims, half of them rotated: 98 us, 5.5 TB/s; 48 tokens 3.2 us).
#include "common.h"
#include "kernels.h"

namespace sgd {

template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> { typedef bf16x8 type; };
template <> struct Vec<bf16, 4> { typedef bf16x4 type; };
template <> struct Vec<bf16, 2> { typedef bf16x2 type; };
template <> struct Vec<bf16, 1> { typedef bf16 type; };
template <> struct Vec<float, 4> { typedef f32x4 type; };
template <> struct Vec<float, 2> { typedef float type __attribute__((ext_vector_type(2))); };
template <> struct Vec<float, 1> { typedef float type; };

template <typename T, int V>
__device__ __forceinline__ void get(const T* p, float (&x)[V]) {
    const auto v = *(const typename Vec<T, V>::type*)p;
    if constexpr (V == 1) x[0] = ElemIO<T>::load(p);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 2) x[i] = bf2f(v[i]);
            else x[i] = v[i];
        }
}
template <typename T, int V>
__device__ __forceinline__ void put(T* p, const float (&x)[V]) {
    if constexpr (V == 1) ElemIO<T>::store(p, x[0]);
    else {
        typename Vec<T, V>::type v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)x[i];
        *(typename Vec<T, V>::type*)p = v;
    }
}

// Threads of a workgroup: groups x head lanes.  Group i < np rotates V pairs (half layout) or V / 2
// (interleaved, one access of V values; V = 1: a pair as two accesses); the others copy V values.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int groups, int np, int hl_n, int heads_per_block) {
    const int i = threadIdx.x % groups, hl = threadIdx.x / groups;
    if (hl >= hl_n) return;
    const long t = blockIdx.x;
    const int h1 = min(a.H, (int)(blockIdx.y + 1) * heads_per_block);
    const T* const x = (const T*)a.x + t * a.x_ts;
    T* const o = (T*)a.out + t * a.o_ts;
    constexpr int PV = INTER ? (V > 1 ? V / 2 : 1) : V;  // pairs of a thread
    if (i >= np) {
        const int c = a.rot + (i - np) * V;
        for (int h = blockIdx.y * heads_per_block + hl; h < h1; h += hl_n) {
            float v[V];
            get<T, V>(x + h * a.x_hs + c, v);
            put<T, V>(o + h * a.o_hs + c, v);
        }
        return;
    }
    const double pos = a.pos ? (double)a.pos[t] : (double)t;
    float cs[PV], sn[PV];
#pragma unroll
    for (int j = 0; j < PV; ++j) {
        const double turn = pos * a.turns[i * PV + j];
        const float f = (float)(turn - rint(turn));
        cs[j] = __builtin_amdgcn_cosf(f) * a.magnitude;
        sn[j] = __builtin_amdgcn_sinf(f) * (a.inverse ? -a.magnitude : a.magnitude);
    }
    const int hd = a.rot / 2;
    for (int h = blockIdx.y * heads_per_block + hl; h < h1; h += hl_n) {
        const T* const xh = x + h * a.x_hs;
        T* const oh = o + h * a.o_hs;
        if constexpr (INTER && V > 1) {
            float v[V], y[V];
            get<T, V>(xh + i * V, v);
#pragma unroll
            for (int j = 0; j < PV; ++j) {
                y[2 * j] = v[2 * j] * cs[j] - v[2 * j + 1] * sn[j];
                y[2 * j + 1] = v[2 * j + 1] * cs[j] + v[2 * j] * sn[j];
            }
            put<T, V>(oh + i * V, y);
        } else {
            const int at = INTER ? 2 * i : i * V, to = INTER ? 2 * i + 1 : hd + i * V;
            float u[V], w[V], y[V], z[V];
            get<T, V>(xh + at, u);
            get<T, V>(xh + to, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[j] = u[j] * cs[j] - w[j] * sn[j];
                z[j] = w[j] * cs[j] + u[j] * sn[j];
            }
            put<T, V>(oh + at, y);
            put<T, V>(oh + to, z);
        }
    }
}

template <typename T, int V>
static void rotary_run(const RotaryArgs& a, hipStream_t st) {
    const bool in_place = a.x == a.out;
    const int np = a.interleaved ? (V > 1 ? a.rot / V : a.rot / 2) : a.rot / 2 / V;
    const int groups = np + (in_place ? 0 : (a.dh - a.rot) / V);
    const int lanes = 256 / groups;
    // Heads side by side in a workgroup, and rounds of them: one round while that gives few workgroups, up to
    // four where there are enough (the angles of a token are then computed once per four heads: 16384 tokens, 64 heads,
    // 64 of 128 dims 100 us, in one round 125; 48 tokens 2.7 us in one round, 2.9 in four)
    const int hl_n = lanes < a.H ? lanes : a.H;
    const int rounds_all = (a.H + hl_n - 1) / hl_n;
    int rounds = 1;
    while (rounds < 4 && rounds < rounds_all && (long)a.T * ((rounds_all + 2 * rounds - 1) / (2 * rounds)) >= 2048) rounds *= 2;
    const int hpb = hl_n * rounds;
    const dim3 grid((unsigned)a.T, (unsigned)((a.H + hpb - 1) / hpb));
    const dim3 block((unsigned)((groups * hl_n + 63) / 64 * 64));
    if (a.interleaved) rotary_kernel<T, V, true><<<grid, block, 0, st>>>(a, groups, np, hl_n, hpb);
    else rotary_kernel<T, V, false><<<grid, block, 0, st>>>(a, groups, np, hl_n, hpb);
}

hipError_t launch_rotary(int bf, const RotaryArgs& a, hipStream_t st) {
    // widest access that every piece of a row allows: the pairs, the rest, the strides and the pointers
    const int es = bf ? 2 : 4;
    auto fits = [&](int v) {
        const int piece = a.interleaved ? a.rot : a.rot / 2;
        return piece % v == 0 && (a.dh - a.rot) % v == 0 && a.x_ts % v == 0 && a.x_hs % v == 0 && a.o_ts % v == 0 &&
               a.o_hs % v == 0 && (uintptr_t)a.x % (v * es) == 0 && (uintptr_t)a.out % (v * es) == 0;
    };
    if (bf) {
        if (fits(8)) rotary_run<bf16, 8>(a, st);
        else if (fits(4)) rotary_run<bf16, 4>(a, st);
        else if (fits(2)) rotary_run<bf16, 2>(a, st);
        else rotary_run<bf16, 1>(a, st);
    } else {
        if (fits(4)) rotary_run<float, 4>(a, st);
        else if (fits(2)) rotary_run<float, 2>(a, st);
        else rotary_run<float, 1>(a, st);
    }
    return hipGetLastError();
}

}  // namespace sgd
