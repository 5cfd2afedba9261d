/*
 * sgd_ops.h -- single-kernel entry points of libsgd.  The first part, up to the microscaled rows, is
 * for kernel-level parity tests and microbenchmarks: exactly the kernels that sgd_denoise_step launches.  The
 * second part are operators of units beyond it: rows in 8 and 4 bits and their products, rotary positions,
 * attention over key intervals.
 *
 * Conventions as in sgd.h: int status (SGD_OK or SGD_E_*), device pointers, enqueue on
 * hip_stream without synchronising, caller-owned buffers, no allocation.
 */
#ifndef SGD_OPS_H
#define SGD_OPS_H

#include <stdint.h>

#include "sgd.h"

#ifdef __cplusplus
extern "C" {
#endif

enum sgd_act { SGD_ACT_NONE = 0, SGD_ACT_GELU_ERF = 1, SGD_ACT_GELU_TANH = 2, SGD_ACT_SILU = 3 };

/* out[M x N] = act(A[M x K] W[N x K]^T + bias) in dtype (the branch GEMM of an MLP input
 * projection).  gated != 0: W is [2N x K] = [W_gate; W_up] and out = act(A W_gate^T +
 * b[:N]) * (A W_up^T + b[N:]).  lda/ldw/ldo are row strides in elements.  tile selects a
 * bf16 kernel variant (0 auto; 1..7 fixed block tiles, for tests and sweeps: 1 256x256,
 * 2 256x128, 3 128x256, 4 128x128, 5 256x192, 6 128x64, 7 64x64, rows x columns).  Shape limits (bf16): K % 64 == 0,
 * N % 4 == 0, gated N a multiple of the tile width, operand rows and bias 16-byte aligned;
 * (fp32): K % 16 == 0, N % 64 == 0. */
int sgd_op_linear(int32_t dtype, const void* A, int64_t lda, const void* W, int64_t ldw, const float* bias,
                  void* out, int64_t ldo, int32_t M, int32_t N, int32_t K, int32_t act, int32_t gated,
                  int32_t tile, void* hip_stream);

/* Attention (Sec. 3 units; the softmax(q k^T / sqrt(dh)) v of every head).  q [B*H, npq, dh],
 * k [B*H, npk, dh], vt [B*H, dh, npk] (dtype), o [B, nq, H*dh].  Keys >= nk are masked;
 * npk must be a multiple of 64 and >= nk; npq >= nq; 8 <= dh <= 128, dh % 8 == 0.  q, k, vt
 * 16-byte aligned, o 16-byte (fp32) or 8-byte (bf16) aligned. */
int sgd_op_attention(int32_t dtype, const void* q, const void* k, const void* vt, void* o, int32_t B, int32_t H,
                     int32_t dh, int32_t nq, int32_t npq, int32_t nk, int32_t npk, void* hip_stream);

/* Pre-norm of M rows of width d from fp32 x into y (dtype).  kind 0: RMSNorm with gain w;
 * 1: LayerNorm with gain w and shift b; 2: LayerNorm without affine parameters followed by
 * y * (1 + scale[r / ntok]) + shift[r / ntok] (rows of scale/shift mod_ld apart).  x, w, b,
 * shift, scale 16-byte aligned (mod_ld % 4 == 0), y 16-byte (fp32) or 8-byte (bf16) aligned. */
int sgd_op_norm(int32_t dtype, int32_t kind, const float* x, void* y, int32_t M, int32_t d, float eps,
                const float* w, const float* b, const float* shift, const float* scale, int64_t mod_ld,
                int32_t ntok, void* hip_stream);

/* The pre-norm that absorbs a frozen run (what the launcher runs when a run of frozen units
 * ends at an active unit, Sec. 3.1 frozen rule): x <- x + deltas[0] + ... + deltas[r-1],
 * added in that order and written back to x (fp32 [M x d], the residual stream), then y = the
 * pre-norm of the new x exactly as sgd_op_norm computes it.  1 <= r <= 32; deltas: r device
 * pointers (host array) to fp32 [M x d], 16-byte aligned.  Bitwise the same as
 * sgd_op_frozen_run followed by sgd_op_norm. */
int sgd_op_norm_fold(int32_t dtype, int32_t kind, float* x, void* y, int32_t M, int32_t d, float eps,
                     const float* w, const float* b, const float* shift, const float* scale, int64_t mod_ld,
                     int32_t ntok, const float* const* deltas, int32_t r, void* hip_stream);

/* Projection into attention heads (the QKV GEMM of a unit): P = A[M x K] W[n_proj*d x K]^T
 * (+ bias), column n of P belongs to projection which0 + n / d (0: q, 1: k, 2: v^T), head
 * (n % d) / dh, dim n % dh; row r is token r % ntok of sample r / ntok.  q, k are
 * [B*H, np, dh], vt is [B*H, dh, np].  rope != 0 rotates the q and k pairs (i, i + dh/2) of
 * token t by t * 10000^(-2i/dh) (rotary position embedding, the LLaDA attention; bf16 only,
 * dh a multiple of 8; any tile width).  Padded tokens (>= ntok) are not written.  tile as for
 * sgd_op_linear. */
int sgd_op_heads(int32_t dtype, const void* A, const void* W, const float* bias, void* q, void* k, void* vt,
                 int32_t M, int32_t K, int32_t n_proj, int32_t which0, int32_t ntok, int32_t np, int32_t H,
                 int32_t dh, int32_t rope, int32_t tile, void* hip_stream);

/* Residual projection of a branch (the O and W2 GEMMs): v = (A[M x K] W[N x K]^T + bias),
 * v *= gate[r / ntok] if gate != NULL (rows gate_ld apart), then h += v (fp32 [M x N]);
 * delta_mode 1 stores v into delta, 2 adds v to delta (the cached update of Sec. 3.1).  tile as
 * for sgd_op_linear. */
int sgd_op_residual(int32_t dtype, const void* A, int64_t lda, const void* W, const float* bias, float* h,
                    float* delta, int32_t delta_mode, const float* gate, int64_t gate_ld, int32_t ntok,
                    int32_t M, int32_t N, int32_t K, int32_t tile, void* hip_stream);

/* A residual projection in K ranges (the MLP output GEMM of a long-K unit, whose partial
 * products the next pre-norm adds to the stream; Sec. 3.1's update h + F(h) taken in parts):
 * parts + s * part_stride receives the fp32 [M x N] product of A's and W's columns
 * [s K / ksplit, (s + 1) K / ksplit), plus the bias in range 0, for s < ksplit.  bf16 only;
 * K a multiple of 64 ksplit, 2 <= ksplit <= 8, part_stride >= M N (a multiple of 4). */
int sgd_op_linear_split(int32_t dtype, const void* A, const void* W, const float* bias, float* parts,
                        int64_t part_stride, int32_t M, int32_t N, int32_t K, int32_t ksplit, void* hip_stream);
/* The same on a fixed block tile: 0 auto, or 2, 4, 6, 7 (numbered as for sgd_op_linear). */
int sgd_op_linear_split_tile(int32_t dtype, const void* A, const void* W, const float* bias, float* parts,
                             int64_t part_stride, int32_t M, int32_t N, int32_t K, int32_t ksplit, int32_t tile,
                             void* hip_stream);

/* h <- h + delta[0] + ... + delta[r-1] elementwise over n fp32 values (n % 4 == 0), in
 * that order (the frozen-unit update of Sec. 3.1 for a run of r frozen units). */
int sgd_op_frozen_run(float* h, const float* const* deltas, int32_t r, int64_t n, void* hip_stream);

/* DiT AdaLN modulation (Sec. 4.2: conditioning keeps propagating; the per-block shift,
 * scale and gate vectors): mod[b, j] = sum_k x[b, k] W[j, k] + bias[j] for B rows of
 * x = SiLU(c) (fp32 [B x d]), W[n_out x d] of dtype (F32 or BF16), bias fp32 [n_out] or NULL,
 * mod fp32 [B x n_out].  d % 64 == 0; x, W 16-byte aligned.  fp32 accumulation of the exact
 * fp32 products x[b, k] W[j, k]. */
int sgd_op_adaln_mod(int32_t dtype, const float* x, const void* W, const float* bias, float* mod, int32_t B,
                     int32_t d, int32_t n_out, void* hip_stream);

/* SDXL UNet ResNet block: y = SiLU(GroupNorm(x) w + b) in bf16 for x [B, N, C] of dtype
 * in_dtype (the fp32 stream or a bf16 convolution output); groups of C / groups consecutive
 * channels (a multiple of 4) normalised over all N positions of a sample (biased variance,
 * eps), then the per-channel gain w and shift b (fp32 [C]).  C <= 4096.  scratch: caller
 * device memory of sgd_op_group_norm_scratch_bytes (per-block partial sums and the group
 * statistics).  x, w, b, scratch 16-byte aligned, y 8-byte aligned. */
int sgd_op_group_norm_scratch_bytes(int32_t B, int32_t N, int32_t groups, size_t* bytes);
int sgd_op_group_norm_silu(int32_t in_dtype, const void* x, void* y, int32_t B, int32_t N, int32_t C,
                           int32_t groups, float eps, const float* w, const float* b, void* scratch,
                           size_t scratch_bytes, void* hip_stream);

/* 3x3 convolution, stride 1, zero padding 1, of bf16 A [M x Cin] holding M / side^2 row-major
 * side x side grids, with the bf16 kernel W [N x 9 Cin] unfolded tap-major (column
 * (3 ky + kx) Cin + c multiplies channel c at grid offset (ky - 1, kx - 1)), as an implicit
 * GEMM on the matrix cores.  h == NULL: out [M x N] bf16 = conv + bias + rowbias[sample]
 * (rowbias fp32 [M / side^2 x N] or NULL); h != NULL: h [M x N] fp32 += conv + bias.
 * Cin % 64 == 0, N % 4 == 0.  tile: 0 auto, or 2, 4, 5, 6, 7 (numbered as for sgd_op_linear). */
int sgd_op_conv3x3(const void* A, const void* W, const float* bias, const float* rowbias, int32_t side, void* out,
                   float* h, int32_t M, int32_t N, int32_t Cin, int32_t tile, void* hip_stream);

/* ------------------------------------------------------------ microscaled rows
 * Rows in 8 or 4 bits with one power-of-two scale per 32 columns (the OCP Microscaling formats):
 *   codes   SGD_MX_FP8: e4m3, one byte a value, K bytes a row; SGD_MX_FP4: e2m1, K / 2 bytes a row, the
 *           even column in the low four bits.  Rows are compact (no row stride).
 *   scales  one byte per row and 32 columns, 2^(byte - 127), 255: NaN; in chunks of eight blocks,
 *           [ceil(K / 256)][rows][8]: byte (c, r, i) is block 8 c + i of row r.  Bytes past the last
 *           block (K % 256 != 0) are written as 0; whoever makes scales must not leave 255 there.
 * Quantisation of a block: scale 2^(floor(log2(max |x|)) - e), e = 8 (e4m3) or 2 (e2m1), not below 2^-127; each
 * x / scale rounded to nearest, ties to even, saturating at 448 or 6 (at most an eighth, or a quarter,
 * off the block's largest values).  A block that holds an infinity or a NaN gets scale 255.
 * K % 32 == 0, codes 16-byte and scales 8-byte aligned. */
enum sgd_mx_format { SGD_MX_FP8 = 0, SGD_MX_FP4 = 1 };

/* Bytes of the codes and scales of `rows` rows of K columns. */
int sgd_op_mx_bytes(int32_t format, int64_t rows, int32_t K, size_t* codes, size_t* scales);

/* x [rows x K] of dtype, rows ldx elements apart (16-byte aligned rows), to codes and scales;
 * rows * K < 2^34. */
int sgd_op_mx_quantize(int32_t format, int32_t dtype, const void* x, int64_t ldx, int32_t rows, int32_t K,
                       void* codes, uint8_t* scales, void* hip_stream);
/* The values back: out [rows x K] of dtype (exact in fp32; in bf16 but for results past its range). */
int sgd_op_mx_dequantize(int32_t format, const void* codes, const uint8_t* scales, int32_t rows, int32_t K,
                         int32_t dtype, void* out, int64_t ldo, void* hip_stream);

/* sgd_op_linear on microscaled rows: out = act(A W^T + bias) with A [M x K] in a_format and W [N x K] (gated:
 * [2N x K] = [W_gate; W_up]) in SGD_MX_FP4.  out_dtype SGD_BF16, or SGD_F32 (ungated, act SGD_ACT_NONE); rows of
 * out ldo elements apart.  Products are summed in fp32.  With A in e2m1 they are exact; with A in e4m3 the matrix
 * cores add those of eight neighbouring columns cut 13 bits below the group's largest exponent (also for fp32 output), which
 * takes nothing where a group's elements of A lie within eight binades.  Of sqrt(sum (a w)^2): rows quantised from normal
 * values 4e-6 on average, 4e-5 at most; codes from all of e4m3 5e-5 and 3e-4.  tile: 0 auto, 1..7 block tiles (256x256, 256x192, 256x128,
 * 128x256, 128x128, 128x64, 64x64), 8 the kernel for up to 16 rows.  N % 4 == 0 (gated: N % 32 == 0, and on a fixed
 * tile 2N a multiple of its width), bias 16-byte, out 8-byte (fp32: 16-byte) aligned, ldo % 4 == 0, each
 * operand's scales and W's codes below 4 GiB, K <= 2^22, fewer than 2^23 tiles.  out overlaps no operand. */
int sgd_op_linear_mx(int32_t a_format, const void* a_codes, const uint8_t* a_scales, const void* w_codes,
                     const uint8_t* w_scales, const float* bias, int32_t out_dtype, void* out, int64_t ldo,
                     int32_t M, int32_t N, int32_t K, int32_t act, int32_t gated, int32_t tile, void* hip_stream);

/* The pre-norm that adds a branch's output to the stream and writes 8- or 4-bit rows: h = x + add (fp32
 * sum, held in x's type), xo = h, codes and scales = h / sqrt(mean(h^2) + eps) w.  x, xo [M x d] of x_dtype
 * (xo may be x), add [M x d] of add_dtype or NULL (then h = x and xo is not written; it may be NULL).  The
 * norm is evaluated in fp64 and rounded once (past fp32's range it counts as infinite).  M < 2^24, d % 32 == 0, d <= 8192; x, add, xo, w 16-byte aligned, none
 * of them overlapping codes or scales. */
int sgd_op_norm_add_mx(int32_t format, int32_t x_dtype, const void* x, int32_t add_dtype, const void* add, void* xo,
                       const float* w, float eps, int32_t M, int32_t d, void* codes, uint8_t* scales, void* hip_stream);

/* ------------------------------------------------------------ rotary positions */

/* How the rotation speeds of a head's pairs are scaled for contexts longer than the model's own.
 *   SGD_ROPE_PLAIN   base^(-2 i / rot) radians a token for pair i < rot / 2
 *   SGD_ROPE_LINEAR  all of them divided by factor
 *   SGD_ROPE_BASE    base factor^(rot / (rot - 2)) in place of base (the slowest pair is divided by factor,
 *                    the fastest kept); rot > 2
 *   SGD_ROPE_PARTS   pairs of more than `high` turns over `context` tokens kept, those of fewer than
 *                    `low` divided by factor, in between mixed linearly in the number of turns; the rotated
 *                    dims are also to be multiplied by 0.1 ln(factor) + 1 (the magnitude returned) */
enum sgd_rope_scaling { SGD_ROPE_PLAIN = 0, SGD_ROPE_LINEAR = 1, SGD_ROPE_BASE = 2, SGD_ROPE_PARTS = 3 };
typedef struct {
    double base;      /* 10000 in the LLaDA attention; > 0 */
    int32_t scaling;  /* sgd_rope_scaling */
    double factor;    /* >= 1; not read for SGD_ROPE_PLAIN */
    double context;   /* SGD_ROPE_PARTS: the model's own context, > 0 */
    double low, high; /* SGD_ROPE_PARTS: 0 <= low < high, usually 1 and 32 */
} sgd_rope_params;
/* Host only: turns per token of the rot / 2 pairs (turns: host [rot / 2]) and the magnitude. */
int sgd_rope_turns(const sgd_rope_params* params, int32_t rot, double* turns, double* magnitude);

/* Rotates dims [0, rot) of every head of T tokens by their position and copies the others: x, out [T, H, dh] of
 * dtype, last dim contiguous, token and head strides in elements (out may be x with the same strides; no
 * other overlap).  Pair p is dims (p, p + rot / 2), or with interleaved != 0 (2 p, 2 p + 1); it turns by pos[t]
 * turns[p] (device fp64 [rot / 2], as from sgd_rope_turns, taken in fp64) and is multiplied by magnitude;
 * inverse != 0 turns back (and multiplies: the transpose, which is the gradient).  pos device int32 [T], or NULL:
 * token t is at position t.  rot even, 2 <= rot <= dh <= 256, T < 2^24, H <= 65535. */
int sgd_op_rotary(int32_t dtype, const void* x, int64_t x_token, int64_t x_head, void* out, int64_t out_token,
                  int64_t out_head, int32_t T, int32_t H, int32_t dh, int32_t rot, int32_t interleaved, const int32_t* pos,
                  const double* turns, float magnitude, int32_t inverse, void* hip_stream);

/* ------------------------------------------------------------ attention over key intervals */

/* One call of sgd_op_attention_ranges.  Tensors are rows of dh contiguous values with strides
 * (batch, token, head) in elements: q, o [B, nq, H, dh], k, v [B, nk, Hk, dh]; H / Hk query heads share a key
 * head (query heads h G .. h G + G - 1 belong to key head h, G = H / Hk).
 *   ranges  device int32 [B, nq, 2]: query i of sample b sees the keys lo <= j < hi (clipped to 0 <= j < nk); where
 *           lo >= hi the output is zero.  Packed documents, prefixes, causal order, padding, windows.
 *   scale   factor of the scores (2^-126 to 2^126; 0 selects 1 / sqrt(dh))
 *   cap     0, or > 0 (at most 2^126, bf16: 1024): scores become cap tanh(score / cap); scale / cap from 2^-126 to 2^126
 *   slopes  NULL, or device fp32 [H]: slope |pos - j| is subtracted from the (capped) score of key j
 *   pos     device int32 [B, nq]: the queries' key positions, for slopes; NULL: i + nk - nq
 * 8 <= dh <= 128, dh % 8 == 0; B Hk <= 65535, nk <= 2^30, nq H / Hk <= 2^30 and fewer than 2^24 blocks of 128 such rows in all
 * key heads; q, k, v rows 16-byte aligned (strides of 8 bf16 or 4 fp32 values), o 8-byte
 * (fp32: 16-byte); token strides of k and v at least dh and below 2^24.  Keys and values that no query sees are
 * not used, whatever they hold; infinities and NaN reach only the queries that see them (an infinite value whose
 * weight underflows arrives as infinity or NaN).  The rows of o are apart from each other and from every input. */
typedef struct {
    const void *q, *k, *v;
    void* o;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
    const int32_t* ranges;
    const int32_t* pos;
    const float* slopes;
    int32_t B, H, Hk, dh, nq, nk;
    float scale, cap;
} sgd_range_attention;
/* Device workspace (16-byte aligned) of a call, 0 for most: with few query rows the keys are split between
 * workgroups, whose results meet there.  Nothing in it needs to start at any value; calls that may run at the same
 * time (replays of two graphs among them) need one each. */
int sgd_op_attention_ranges_bytes(int32_t dtype, const sgd_range_attention* call, size_t* bytes);
int sgd_op_attention_ranges(int32_t dtype, const sgd_range_attention* call, void* workspace, size_t workspace_bytes,
                            void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SGD_OPS_H */
