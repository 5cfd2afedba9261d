// C ABI of the operators beyond the step's own kernels (second part of sgd_ops.h): argument checks, then
// one or two launches.  Everything is checked before anything is enqueued.
#include <cfloat>
#include <cmath>

#include "../../include/sgd_ops.h"
#include "internal.h"
#include "kernels.h"

using namespace sgd;

namespace {
bool aligned(const void* p, unsigned a) { return (uintptr_t)p % a == 0; }
bool is_dtype(int32_t d) { return d == SGD_F32 || d == SGD_BF16; }
bool is_format(int32_t f) { return f == SGD_MX_FP8 || f == SGD_MX_FP4; }
int64_t code_bytes(int32_t format, int64_t rows, int64_t K) { return rows * (format == SGD_MX_FP8 ? K : K / 2); }
int64_t scale_bytes(int64_t rows, int64_t K) { return (K + 255) / 256 * rows * 8; }
constexpr int64_t kBuffer = 0xFFFFFF00;  // 32-bit buffer ranges below the loaders' out-of-range offset

int check_mx(int32_t format, int32_t dtype, const void* codes, const uint8_t* scales, const void* x, int64_t ld,
             int32_t rows, int32_t K) {
    if (!codes || !scales || !x) return fail(SGD_E_ARG, "NULL argument");
    if (!is_format(format)) return fail(SGD_E_DTYPE, "format must be MX_FP8 or MX_FP4");
    if (!is_dtype(dtype)) return fail(SGD_E_DTYPE, "dtype must be F32 or BF16");
    if (rows < 1 || K < 32 || K % 32 || (int64_t)rows * K >= (1LL << 34))
        return fail(SGD_E_SHAPE, "microscaled rows: rows >= 1, K a multiple of 32, rows * K < 2^34");
    const int v = dtype == SGD_BF16 ? 8 : 4;
    if (ld < K || ld % v || !aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 8))
        return fail(SGD_E_ARG, "rows must be 16-byte aligned and at least K apart (codes 16-byte, scales 8-byte aligned)");
    return SGD_OK;
}
}  // namespace

extern "C" int sgd_op_mx_bytes(int32_t format, int64_t rows, int32_t K, size_t* codes, size_t* scales) {
    if (!codes || !scales) return fail(SGD_E_ARG, "NULL argument");
    if (!is_format(format)) return fail(SGD_E_DTYPE, "format must be MX_FP8 or MX_FP4");
    if (rows < 1 || rows > INT32_MAX || K < 32 || K % 32) return fail(SGD_E_SHAPE, "rows >= 1, K a multiple of 32");
    *codes = (size_t)code_bytes(format, rows, K);
    *scales = (size_t)scale_bytes(rows, K);
    return SGD_OK;
}

extern "C" int sgd_op_mx_quantize(int32_t format, int32_t dtype, const void* x, int64_t ldx, int32_t rows, int32_t K,
                                  void* codes, uint8_t* scales, void* hip_stream) {
    const int rc = check_mx(format, dtype, codes, scales, x, ldx, rows, K);
    if (rc) return rc;
    MxQuantArgs a;
    a.x = x; a.ldx = ldx; a.rows = rows; a.K = K; a.codes = (uint8_t*)codes; a.scales = scales;
    SGD_HIP_TRY(launch_mx_quantize(format, dtype == SGD_BF16, a, (hipStream_t)hip_stream));
    return SGD_OK;
}

extern "C" int sgd_op_mx_dequantize(int32_t format, const void* codes, const uint8_t* scales, int32_t rows, int32_t K,
                                    int32_t dtype, void* out, int64_t ldo, void* hip_stream) {
    const int rc = check_mx(format, dtype, codes, scales, out, ldo, rows, K);
    if (rc) return rc;
    MxQuantArgs a;
    a.out = out; a.ldx = ldo; a.rows = rows; a.K = K;
    a.codes = (uint8_t*)const_cast<void*>(codes); a.scales = const_cast<uint8_t*>(scales);
    SGD_HIP_TRY(launch_mx_dequantize(format, dtype == SGD_BF16, a, (hipStream_t)hip_stream));
    return SGD_OK;
}

extern "C" int sgd_op_linear_mx(int32_t a_format, const void* a_codes, const uint8_t* a_scales, const void* w_codes,
                                const uint8_t* w_scales, const float* bias, int32_t out_dtype, void* out, int64_t ldo,
                                int32_t M, int32_t N, int32_t K, int32_t act, int32_t gated, int32_t tile,
                                void* hip_stream) {
    if (!a_codes || !a_scales || !w_codes || !w_scales || !out) return fail(SGD_E_ARG, "NULL argument");
    if (!is_format(a_format)) return fail(SGD_E_DTYPE, "a_format must be MX_FP8 or MX_FP4");
    if (!is_dtype(out_dtype)) return fail(SGD_E_DTYPE, "out_dtype must be F32 or BF16");
    if (act < 0 || act > 3 || tile < 0 || tile > kMxTiles) return fail(SGD_E_ARG, "bad act or tile");
    if (out_dtype == SGD_F32 && (gated || act != SGD_ACT_NONE))
        return fail(SGD_E_DTYPE, "fp32 output takes no activation and no gate");
    if (M < 1 || N < 4 || N % 4 || K < 32 || K % 32 || (gated && (N % 32 || N > INT32_MAX / 2)))
        return fail(SGD_E_SHAPE, "M >= 1, N a multiple of 4 (gated: 32), K a multiple of 32");
    const int64_t n = gated ? 2LL * N : N;
    if (code_bytes(SGD_MX_FP4, n + 256, K) > kBuffer ||  // a tile's rows past N must not wrap around
         scale_bytes(n, K) > kBuffer || scale_bytes(M, K) > kBuffer ||
        K > (1 << 22))
        return fail(SGD_E_SHAPE, "W's codes and either scales must be below 4 GiB, K at most 2^22");
    if (ldo < N || ldo % 4 || !aligned(out, out_dtype == SGD_F32 ? 16 : 8) || !aligned(bias, 16) || !aligned(a_codes, 16) ||
        !aligned(w_codes, 16) || !aligned(a_scales, 8) || !aligned(w_scales, 8))
        return fail(SGD_E_ARG, "operands must be aligned as documented, ldo >= N a multiple of 4");
    GemmArgs g;
    g.A0 = a_codes; g.B = w_codes; g.M = M; g.N = (int)n; g.K = K;
    EpiParams e;
    e.bias = bias; e.act = act;
    if (out_dtype == SGD_F32) {
        e.kind = EP_PARTIAL; e.h = (float*)out; e.d = (int)ldo;
    } else {
        e.kind = gated ? EP_GATED : EP_ACT; e.out = out; e.ldo = ldo; e.F = N;
    }
    if (ldo > INT32_MAX || !gemm_mx_shape_ok(a_format, g, e, tile)) return fail(SGD_E_SHAPE, "the tile does not take this shape");
    const MxScales s{a_scales, w_scales};
    SGD_HIP_TRY(launch_gemm_mx(a_format, g, e, s, tile, (hipStream_t)hip_stream));
    return SGD_OK;
}

extern "C" int sgd_op_norm_add_mx(int32_t format, int32_t x_dtype, const void* x, int32_t add_dtype, const void* add,
                                  void* xo, const float* w, float eps, int32_t M, int32_t d, void* codes,
                                  uint8_t* scales, void* hip_stream) {
    if (!x || !w || !codes || !scales || (add && !xo)) return fail(SGD_E_ARG, "NULL argument");
    if (!is_format(format)) return fail(SGD_E_DTYPE, "format must be MX_FP8 or MX_FP4");
    if (!is_dtype(x_dtype) || (add && !is_dtype(add_dtype))) return fail(SGD_E_DTYPE, "dtype must be F32 or BF16");
    if (M < 1 || M >= (1 << 24) || d < 32 || d % 32 || d > 8192)  // a launch has at most 2^32 threads
        return fail(SGD_E_SHAPE, "norm: 1 <= M < 2^24, d a multiple of 32, at most 8192");
    if (!(eps >= 0.f)) return fail(SGD_E_ARG, "eps must not be negative");
    if (!aligned(x, 16) || !aligned(add, 16) || !aligned(xo, 16) || !aligned(w, 16) || !aligned(codes, 16) || !aligned(scales, 8))
        return fail(SGD_E_ARG, "norm operands must be 16-byte aligned (scales: 8)");
    const NormMxArgs a{x, add, xo, w, eps, M, d, (uint8_t*)codes, scales};
    SGD_HIP_TRY(launch_norm_add_mx(format, x_dtype == SGD_BF16, add && add_dtype == SGD_BF16, a, (hipStream_t)hip_stream));
    return SGD_OK;
}

extern "C" int sgd_rope_turns(const sgd_rope_params* p, int32_t rot, double* turns, double* magnitude) {
    if (!p || !turns || !magnitude) return fail(SGD_E_ARG, "NULL argument");
    if (rot < 2 || rot % 2) return fail(SGD_E_SHAPE, "rot must be even");
    if (p->scaling < SGD_ROPE_PLAIN || p->scaling > SGD_ROPE_PARTS) return fail(SGD_E_ARG, "unknown scaling");
    const bool scaled = p->scaling != SGD_ROPE_PLAIN, parts = p->scaling == SGD_ROPE_PARTS;
    if (!(p->base > 0) || !std::isfinite(p->base) || (scaled && (!(p->factor >= 1) || !std::isfinite(p->factor))))
        return fail(SGD_E_ARG, "base must be positive, factor at least 1");
    if (parts && (!(p->context > 0) || !(p->low >= 0) || !(p->high > p->low) || !std::isfinite(p->high) || !std::isfinite(p->context)))
        return fail(SGD_E_ARG, "context must be positive, 0 <= low < high");
    if (p->scaling == SGD_ROPE_BASE && rot < 4) return fail(SGD_E_SHAPE, "a changed base needs rot > 2");
    const double base = p->scaling == SGD_ROPE_BASE ? p->base * std::pow(p->factor, (double)rot / (rot - 2)) : p->base;
    for (int i = 0; i < rot / 2; ++i) {
        double t = std::pow(base, -2.0 * i / rot) / 6.283185307179586476925286766559;
        if (p->scaling == SGD_ROPE_LINEAR) t /= p->factor;
        if (parts) {
            const double keep = std::fmin(1.0, std::fmax(0.0, (t * p->context - p->low) / (p->high - p->low)));
            t = t * keep + t / p->factor * (1.0 - keep);
        }
        turns[i] = t;
    }
    *magnitude = parts ? 0.1 * std::log(p->factor) + 1.0 : 1.0;
    return SGD_OK;
}

extern "C" int sgd_op_rotary(int32_t dtype, const void* x, int64_t x_token, int64_t x_head, void* out, int64_t out_token,
                             int64_t out_head, int32_t T, int32_t H, int32_t dh, int32_t rot, int32_t interleaved,
                             const int32_t* pos, const double* turns, float magnitude, int32_t inverse, void* hip_stream) {
    if (!x || !out || !turns) return fail(SGD_E_ARG, "NULL argument");
    if (!is_dtype(dtype)) return fail(SGD_E_DTYPE, "dtype must be F32 or BF16");
    if (T < 1 || T >= (1 << 24) || H < 1 || H > 65535 || dh < 2 || dh > 256 || rot < 2 || rot % 2 || rot > dh)
        return fail(SGD_E_SHAPE, "rotary: 1 <= T < 2^24, 1 <= H <= 65535, 2 <= rot <= dh <= 256, rot even");
    const unsigned es = dtype == SGD_BF16 ? 2 : 4;
    if (!aligned(x, es) || !aligned(out, es) || !aligned(turns, 8) || !aligned(pos, 4))
        return fail(SGD_E_ARG, "rotary operands must be aligned to their elements");
    if ((T > 1 && out_token == 0) || (H > 1 && out_head == 0)) return fail(SGD_E_ARG, "out rows must not coincide");
    if (x == out && ((T > 1 && x_token != out_token) || (H > 1 && x_head != out_head)))
        return fail(SGD_E_ARG, "in place, out has x's strides");
    const RotaryArgs a{x, out, x_token, x_head, out_token, out_head, turns, pos, T, H, dh, rot, interleaved != 0, inverse != 0, magnitude};
    SGD_HIP_TRY(launch_rotary(dtype == SGD_BF16, a, (hipStream_t)hip_stream));
    return SGD_OK;
}

namespace {
// checks a call and turns it into the launcher's arguments
int range_args(int32_t dtype, const sgd_range_attention* c, RangeAttnArgs& a) {
    if (!c) return fail(SGD_E_ARG, "NULL argument");
    if (!is_dtype(dtype)) return fail(SGD_E_DTYPE, "dtype must be F32 or BF16");
    if (c->B < 1 || c->H < 1 || c->Hk < 1 || c->H % c->Hk || c->nq < 1 || c->nk < 1 || c->dh < 8 || c->dh > 128 || c->dh % 8)
        return fail(SGD_E_SHAPE, "attention shape not supported");
    const int64_t G = c->H / c->Hk, rows = c->nq * G;
    if ((int64_t)c->B * c->Hk > 65535 || rows > (1LL << 30) || c->nk > (1 << 30))
        return fail(SGD_E_SHAPE, "B * Hk at most 65535, query rows of a key head and keys at most 2^30");
    if ((int64_t)c->B * c->Hk * ((rows + 127) / 128) >= (1LL << 24)) return fail(SGD_E_SHAPE, "too many query rows");
    const int v = dtype == SGD_BF16 ? 8 : 4, vo = 4;
    for (int i = 0; i < 3; ++i)
        if (c->q_stride[i] % v || c->k_stride[i] % v || c->v_stride[i] % v || c->o_stride[i] % vo)
            return fail(SGD_E_ARG, "strides of q, k and v must be multiples of 16 bytes, of o of 4 values");
    for (int64_t s : {c->k_stride[1], c->v_stride[1]})
        if (c->nk > 1 && (s < c->dh || s >= (1 << 24))) return fail(SGD_E_ARG, "token strides of k and v: dh to 2^24");
    if (!(c->scale >= 0.f) || !std::isfinite(c->scale) || !(c->cap >= 0.f) || !std::isfinite(c->cap))
        return fail(SGD_E_ARG, "scale and cap must be finite and not negative");
    if ((c->B > 1 && c->o_stride[0] == 0) || (c->nq > 1 && c->o_stride[1] == 0) || (c->H > 1 && c->o_stride[2] == 0))
        return fail(SGD_E_ARG, "o's rows must not coincide");
    a.q = c->q; a.k = c->k; a.v = c->v; a.o = c->o;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = c->q_stride[i]; a.ks[i] = c->k_stride[i]; a.vs[i] = c->v_stride[i]; a.os[i] = c->o_stride[i];
    }
    if (c->nk == 1) a.ks[1] = a.vs[1] = c->dh;  // one key: its token stride is never taken
    a.ranges = c->ranges; a.pos = c->pos; a.slopes = c->slopes;
    a.B = c->B; a.H = c->H; a.Hk = c->Hk; a.dh = c->dh; a.nq = c->nq; a.nk = c->nk;
    a.scale = c->scale > 0.f ? c->scale : 1.0f / std::sqrt((float)c->dh);
    a.cap = c->cap;
    // the kernels hold scale and cap times log2(e), and 2 log2(e) scale / cap, as normal fp32 numbers
    if (a.scale < FLT_MIN || a.scale > 0x1p126f || a.cap > 0x1p126f) return fail(SGD_E_ARG, "scale: 2^-126 to 2^126, cap: at most 2^126");
    const float ratio = a.cap > 0.f ? a.scale / a.cap : 1.f;
    if (!std::isfinite(4.0f * ratio) || ratio < FLT_MIN || (dtype == SGD_BF16 && a.cap > 1024.f))
        return fail(SGD_E_ARG, "cap: at most 1024 for bf16, and scale / cap must be a normal fp32 number");
    a.work = nullptr;
    a.splits = range_attention_splits(dtype == SGD_BF16, a);
    return SGD_OK;
}
}  // namespace

extern "C" int sgd_op_attention_ranges_bytes(int32_t dtype, const sgd_range_attention* call, size_t* bytes) {
    if (!bytes) return fail(SGD_E_ARG, "NULL argument");
    RangeAttnArgs a;
    const int rc = range_args(dtype, call, a);
    if (rc) return rc;
    *bytes = range_attention_bytes(a, a.splits);
    return SGD_OK;
}

extern "C" int sgd_op_attention_ranges(int32_t dtype, const sgd_range_attention* call, void* workspace,
                                       size_t workspace_bytes, void* hip_stream) {
    RangeAttnArgs a;
    const int rc = range_args(dtype, call, a);
    if (rc) return rc;
    if (!a.q || !a.k || !a.v || !a.o || !a.ranges) return fail(SGD_E_ARG, "NULL argument");
    if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.o, dtype == SGD_F32 ? 16 : 8) ||
        !aligned(a.ranges, 4) || !aligned(a.pos, 4) || !aligned(a.slopes, 4))
        return fail(SGD_E_ARG, "attention operands must be 16-byte aligned (bf16 output: 8)");
    const size_t need = range_attention_bytes(a, a.splits);
    if (need && (!workspace || workspace_bytes < need)) return fail(SGD_E_ARG, "workspace too small");
    if (need && !aligned(workspace, 16)) return fail(SGD_E_ARG, "workspace must be 16-byte aligned");
    a.work = workspace;
    SGD_HIP_TRY(launch_range_attention(dtype == SGD_BF16, a, (hipStream_t)hip_stream));
    return SGD_OK;
}
