/*
 * ekya_ops.h - op-level entry points of the library's kernels.
 *
 * These expose, one at a time, the layer operations the retraining step is
 * built from (the layers of the ResNet18 edge classifier of section 6.1 and
 * the PyTorch training the paper runs, section 5), so that each kernel can be
 * compared with an independent implementation.  They are synchronous: each
 * call enqueues on `stream`, waits for it, and frees its temporaries.  (The
 * adapter-training operators at the end are not: see there.)
 *
 * Common rules: every tensor pointer is a device pointer owned by the caller;
 * activations are NHWC with element type per `precision` (EKYA_FP32 float,
 * EKYA_BF16 bfloat16); weights and per-channel vectors are fp32.  Channel
 * counts must be multiples of 8 (bf16) or 4 (fp32), except an input channel
 * count of 3 (an image), which is zero-padded internally.  Invalid sizes
 * return EKYA_ERR_INVALID_ARG before any GPU work; HIP failures return
 * EKYA_ERR_HIP.
 */
#ifndef EKYA_OPS_H_
#define EKYA_OPS_H_

#include "ekya.h"

#ifdef __cplusplus
extern "C" {
#endif

/* y[N,P,Q,K] = sum_{c,r,s} x[N, stride*p + r - pad, stride*q + s - pad, c] * w[K][C][R][S]
 * (cross-correlation with zero padding), P = (H + 2 pad - R)/stride + 1. */
ekya_status ekya_op_conv2d(int precision, const void* x, int N, int H, int W, int C,
                           const float* w, int K, int R, int S, int stride, int pad, void* y,
                           void* stream);
/* dx[N,H,W,C]: gradient of ekya_op_conv2d with respect to x for dy[N,P,Q,K]. */
ekya_status ekya_op_conv2d_dgrad(int precision, const void* dy, const float* w, int N, int H,
                                 int W, int C, int K, int R, int S, int stride, int pad, void* dx,
                                 void* stream);
/* dw[K][C][R][S] (fp32): gradient of ekya_op_conv2d with respect to w. */
ekya_status ekya_op_conv2d_wgrad(int precision, const void* x, const void* dy, int N, int H,
                                 int W, int C, int K, int R, int S, int stride, int pad,
                                 float* dw, void* stream);
/* Train-mode BatchNorm over z[M, C] (M = N*H*W rows): y = gamma*(z-mean)*invstd
 * + beta (then ReLU if relu), biased batch variance, eps 1e-5; running
 * statistics (optional, may be null) updated with momentum 0.1 and the
 * unbiased variance.  mean_out/invstd_out: [C] fp32. */
ekya_status ekya_op_batchnorm_train(int precision, const void* z, long long M, int C,
                                    const float* gamma, const float* beta, float* running_mean,
                                    float* running_var, int relu, void* y, float* mean_out,
                                    float* invstd_out, void* stream);
/* ekya_op_batchnorm_train for callers that cannot allocate device memory
 * (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): same arguments, kernels and results (bitwise), but it calls no
 * hipMalloc / hipFree and does not synchronise -- the work is queued on
 * `stream` and the caller synchronises.  Its scratch (partial sums, scale and
 * shift) is one static device array per GPU of 512*2*2048 + 5*2048 floats
 * (about 8.4 MB), enough for every M and C <= 2048; a request that would
 * need more returns EKYA_ERR_INVALID_ARG.  The first call on a device looks
 * up the array's address (make it outside graph capture).  Every call on one
 * GPU shares that array, so calls that overlap on one GPU (different
 * streams without ordering between them) race; nothing in it needs to start
 * at zero. */
ekya_status ekya_op_batchnorm_train_noalloc(int precision, const void* z, long long M, int C,
                                            const float* gamma, const float* beta,
                                            float* running_mean, float* running_var, int relu,
                                            void* y, float* mean_out, float* invstd_out,
                                            void* stream);
/* Backward of ekya_op_batchnorm_train: g = dy * [y_relu > 0] (no mask when
 * y_relu is null); dbeta = sum g, dgamma = sum g*xhat,
 * dz = gamma*invstd/M*(M*g - dbeta - xhat*dgamma). */
ekya_status ekya_op_batchnorm_backward(int precision, const void* dy, const void* y_relu,
                                       const void* z, long long M, int C, const float* gamma,
                                       const float* mean, const float* invstd, void* dz,
                                       float* dgamma, float* dbeta, void* stream);
/* 3x3 stride-2 pad-1 max pooling (padding never wins); arg[N,P,Q,C] (uint8)
 * is the row-major window index of the first maximal element. */
ekya_status ekya_op_maxpool(int precision, const void* x, int N, int H, int W, int C, void* y,
                            uint8_t* arg, void* stream);
ekya_status ekya_op_maxpool_backward(int precision, const void* dy, const uint8_t* arg, int N,
                                     int H, int W, int C, void* dx, void* stream);
/* f[N, C] (fp32) = mean of x over H*W; and its backward dx = df / (H*W). */
ekya_status ekya_op_avgpool(int precision, const void* x, int N, int H, int W, int C, float* f,
                            void* stream);
ekya_status ekya_op_avgpool_backward(int precision, const float* df, int N, int H, int W, int C,
                                     void* dx, void* stream);
/* Classifier: z[N,J] = f[N,I] W[J,I]^T + b, and its backward (fp32). */
ekya_status ekya_op_linear(const float* f, const float* Wt, const float* b, int N, int I, int J,
                           float* z, void* stream);
ekya_status ekya_op_linear_backward(const float* dz, const float* f, const float* Wt, int N,
                                    int I, int J, float* dW, float* db, float* df, void* stream);
/* Mean softmax cross-entropy of z[N,J] against labels[N]: dz = (softmax -
 * onehot)/N; out[0] = mean loss, out[1] = correct count, out[2] = non-finite
 * flag (device fp32 [3]). */
ekya_status ekya_op_softmax_ce(const float* z, const int32_t* labels, int N, int J, float* dz,
                               float* out, void* stream);
/* SGD with momentum over n floats: v = mu v + g; w = w - lr v. */
ekya_status ekya_op_sgd(float* w, float* v, const float* g, long long n, float lr, float mu,
                        void* stream);
/* Bilinear resize (half-pixel centres, clamped at 0, no antialiasing) of
 * frames [n,H,W,3] to [n,r,r,3]. */
ekya_status ekya_op_resize(int precision, const void* frames, int n, int H, int W, int r,
                           void* out, void* stream);

/* ------------------------------------------------- adapter-training operators
 * What fine-tuning an adapter or a head on the network's features needs beside
 * the layers above: group norm in place of BatchNorm (whose batch statistics
 * say little on a few frames), matrix products in the activations' type with
 * everything elementwise behind them in the same pass, and AdamW.
 *
 * These calls are asynchronous: they queue kernels on `stream` (of the current
 * device), allocate nothing, copy nothing and never wait, so they can be
 * captured into a HIP graph.  Scratch memory is the caller's: `workspace`, at
 * least as many bytes as the matching *_workspace query says (host only, 0 if
 * an argument is invalid; a query that takes the call's arguments looks at their
 * addresses too), on 16 bytes, written before it is read, free for
 * other use once the call's work has run; calls that may overlap on the GPU,
 * and graphs that may, need one each.  Types per `precision` as above; any
 * channel count, size and alignment to the element is accepted.  Results do
 * not depend on other work on the GPU: every sum has a fixed order. */
typedef enum {
  EKYA_ACT_NONE = 0,
  EKYA_ACT_RELU = 1, /* max(u, 0); derivative 0 at 0 */
  EKYA_ACT_SILU = 2, /* u / (1 + exp(-u)) */
  EKYA_ACT_GELU = 3  /* u (1 + erf(u / sqrt 2)) / 2 */
} ekya_act;

/* Group norm of x[N, HW, C], channels last: the C channels form `groups`
 * groups of C / groups consecutive ones, and each (sample, group) is
 * normalised by its own mean and biased variance over HW * C / groups
 * elements: u = (x - mean) * rstd * gamma + beta, rstd = 1 / sqrt(var + eps),
 * y = act(u).  gamma and beta [C] fp32, both or neither (null: 1 and 0).
 * mean, rstd: [N, groups] fp32 outputs, read by the backward pass.  y may be x;
 * otherwise no output overlaps an input or another output.  N >= 0 (0: nothing
 * is done), HW >= 1, C in [1, 65536], N * HW * C <= 2^40, eps > 0. */
size_t ekya_op_groupnorm_workspace(int precision, int N, long long HW, int C, int groups);
ekya_status ekya_op_groupnorm(int precision, const void* x, int N, long long HW, int C, int groups,
                              const float* gamma, const float* beta, float eps, int act, void* y,
                              float* mean, float* rstd, void* workspace, size_t workspace_bytes,
                              void* stream);
/* Its gradient: with g = dy * act'(u), dbeta = sum g and dgamma = sum g * xhat
 * over samples and pixels, h = g * gamma and dx = rstd * (h - avg(h) -
 * xhat * avg(h * xhat)), averages over the (sample, group).  dgamma and dbeta
 * [C] fp32, both or neither; N = 0 makes them zero.  dx may be dy or x;
 * otherwise no output overlaps an input or another output.  gamma, beta, mean and
 * rstd as the forward call had and returned them. */
size_t ekya_op_groupnorm_backward_workspace(int precision, int N, long long HW, int C, int groups);
ekya_status ekya_op_groupnorm_backward(int precision, const void* dy, const void* x, int N,
                                       long long HW, int C, int groups, const float* gamma,
                                       const float* beta, const float* mean, const float* rstd,
                                       int act, void* dx, float* dgamma, float* dbeta,
                                       void* workspace, size_t workspace_bytes, void* stream);

/* Matrix product with its epilogue: s = x w^T + bias, y = act(s) + residual,
 * or, with residual_first, s = x w^T + bias + residual, y = act(s) (the order
 * of a residual block).  Rows of a matrix are `ld` elements apart, ld >= its
 * width; what lies between them is neither read nor written.  Products are
 * summed in fp32; y and z are rounded once, from that.  Outputs overlap
 * nothing else, but for y, which may be the residual (same start, same ld);
 * columns of one buffer are fine where the lds are equal.  M times the larger
 * of N and K is at most 2^40. */
typedef struct {
  int precision;        /* of x, w, residual, y and z */
  long long M;          /* rows, >= 0 (0: nothing is done) */
  int N, K;             /* outputs and inputs of a row, in [1, 2^24] */
  const void* x;        /* [M][K] */
  long long ldx;
  const void* w;        /* [N][K] */
  long long ldw;
  const float* bias;    /* [N] fp32, or null */
  int act;              /* ekya_act */
  const void* residual; /* [M][N], or null */
  long long ldr;
  int residual_first;
  void* y;              /* [M][N] */
  long long ldy;
  void* z;              /* [M][N], or null: receives s, which the backward pass reads */
  long long ldz;
} ekya_matmul_args;
size_t ekya_op_matmul_workspace(const ekya_matmul_args* args);
ekya_status ekya_op_matmul(const ekya_matmul_args* args, void* workspace, size_t workspace_bytes,
                           void* stream);

/* Its gradient.  dz = dy * act'(z) is the gradient of s (and of the residual
 * where it was added first; otherwise the residual's is dy): dx = dz w, dw =
 * dz^T x, db = sum over rows of dy * act'(z).  dz is stored in `precision` and
 * the products read it as stored; db is summed before that rounding.  With
 * EKYA_ACT_NONE dz is dy: z and dz are not used.  Any of dx, dw, db may be
 * null (x is read for dw only, w for dx only).  M = 0 makes dw and db zero.
 * Overlaps as above: dz may be dy or z. */
typedef struct {
  int precision;    /* of dy, z, x, w, dz and dx */
  long long M;
  int N, K;
  const void* dy;   /* [M][N] */
  long long lddy;
  const void* z;    /* [M][N], as stored by ekya_op_matmul */
  long long ldz;
  int act;
  const void* x;    /* [M][K] */
  long long ldx;
  const void* w;    /* [N][K] */
  long long ldw;
  void* dz;         /* [M][N]; may be dy or z (with its ld) */
  long long lddz;
  void* dx;         /* [M][K] */
  long long lddx;
  void* dw;         /* [N][K], rows next to each other */
  int dw_precision; /* EKYA_FP32, or `precision` */
  float* db;        /* [N] fp32 */
} ekya_matmul_backward_args;
size_t ekya_op_matmul_backward_workspace(const ekya_matmul_backward_args* args);
ekya_status ekya_op_matmul_backward(const ekya_matmul_backward_args* args, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* AdamW over a list of tensors.  For every element, with t = step:
 *   m = beta1 m + (1 - beta1) g          v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 * w is fp32; g is fp32 or bf16; `low`, where given, receives w rounded to bf16
 * (the copy that ekya_op_matmul reads).
 * state_bits 32: m and v are fp32 [n].
 * state_bits 8: m holds n e4m3 and v n e5m2 bytes (OCP formats); element i
 * stands for its byte's value times scale[2 (i / 256)] (m) or
 * scale[2 (i / 256) + 1] (v), fp32 powers of two that a step rewrites: the
 * largest finite value of the block then lies in [128, 256) or [2^14, 2^15) of
 * its scale (a scale is at least 2^-126).  The step rounds the new states
 * stochastically, since rounding to nearest would leave v where it is (beta2
 * = 0.999 moves it by a thousandth, half a unit of e5m2 is an eighth): a
 * magnitude goes up with the probability of its remainder.  The 16 random bits
 * of element i of the list are bits 16 (i mod 4) .. of output i / 4 of the
 * SplitMix64 stream that starts at seed + step * 0xD1B54A32D192ED03, elements
 * counted from one tensor to the next with every tensor filled up to a
 * multiple of 256; v takes their complement.  A v above zero is never rounded
 * to zero (w would move by lr / eps).  Non-finite states are stored as NaN and
 * stay out of their block's scale.  New states are zero bytes with any finite
 * scale. */
typedef struct {
  float* w;
  const void* g;
  void* m;
  void* v;
  float* scale;   /* [2 * ceil(n / 256)] (state_bits 8), else null */
  void* low;      /* bf16 [n], or null */
  long long n;    /* 0 .. 2^38 elements */
  float weight_decay; /* >= 0 */
} ekya_adamw_tensor;
typedef struct {
  double lr, beta1, beta2, eps; /* lr >= 0, betas in [0, 1), eps >= 0 */
  long long step;               /* 1, 2, ...; used where step_device is null */
  const int64_t* step_device;   /* device, or null: the step's number is read on the GPU when
                                   the kernels run, so that a replayed graph can count on;
                                   below 1 it counts as 1 */
  uint64_t seed;                /* stochastic rounding (state_bits 8) */
} ekya_adamw_opts;
typedef struct ekya_adamw ekya_adamw;
/* The list is checked and kept (host memory only); the tensors stay the
 * caller's.  count 0 .. 65536.  EKYA_ERR_INVALID_ARG where a tensor that a step
 * writes overlaps another of the list.  Steps of one handle may be queued from
 * several threads; set_grads needs the handle to itself. */
ekya_status ekya_adamw_create(ekya_adamw** out, const ekya_adamw_tensor* tensors, int count,
                              int grad_precision, int state_bits);
void ekya_adamw_destroy(ekya_adamw* opt);
/* New gradient tensors (count and sizes as created).  A step takes those that
 * are set when it is called. */
ekya_status ekya_adamw_set_grads(ekya_adamw* opt, const void* const* grads, int count);
/* One step over every tensor, asynchronous on `stream`, no workspace. */
ekya_status ekya_adamw_step(const ekya_adamw* opt, const ekya_adamw_opts* opts, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EKYA_OPS_H_ */
