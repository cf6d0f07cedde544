/*
 * hf.h - C ABI of the MI355X (gfx950) Hessian-free curvature library.
 *
 * The library computes, for a fully connected network with sigmoid, tanh or
 * ReLU hidden units and a softmax cross-entropy output averaged over the
 * minibatch:
 *   - the objective f and gradient g_k = grad f(theta_k)       (Alg. 1, step 1)
 *   - curvature-vector products: the exact Hessian H v by the R-operator and
 *     the Gauss-Newton G v                       (Sec. 2.1, after Alg. 1)
 *   - CG-Minimize of the quadratic model m_k(d) = f + g^T d + d^T B_k d / 2
 *     with B_k(d) = A d + lambda d, A = H or G   (Alg. 1 steps 3-4, eq. (1)),
 *     stopping at the first conjugate direction with p^T B_k p <= 0 and
 *     returning the current iterate (or -g at the first iteration) and the
 *     oriented direction d~ = -sgn(g^T p) p      (Sec. 2.1 after eq. (1); Sec. 2.2)
 * on one GPU's share of a data-parallel minibatch (Alg. 2).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Parameter layout (theta, v, g, H v, step, neg_dir): for l = 1..L the
 *   weight matrix W_l (d_l x d_{l-1}, row-major) followed by the bias b_l
 *   (d_l); n = sum_l d_l (d_{l-1} + 1) fp32 values.
 * X: B x d_0 row-major fp32.  y: B int32 labels in [0, d_L).
 * Every array argument is a device pointer, 16-byte aligned, owned by the
 *   caller; the library never allocates or frees device memory.  Scratch
 *   space comes from one caller-provided workspace (hf_set_workspace).
 * All device work is enqueued on the context's stream (hf_create's
 *   hip_stream, changed later with hf_set_stream; NULL = the null stream).
 *   hf_loss_grad and hf_hvp are asynchronous; hf_cg returns after its solve
 *   has finished (it synchronises the stream).
 * Return value: HF_OK or a negative HF_E* code; hf_last_error() gives the
 *   message.  Arguments are validated before any device call, so a bad
 *   argument never reaches the GPU.  No exception or abort crosses the ABI.
 * A context is not thread-safe; calls on one context must not overlap.
 */
#ifndef HF_H
#define HF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hf_ctx hf_ctx;

/* Hidden-layer activation; the output layer is always softmax. */
enum { HF_SIGMOID = 0, HF_TANH = 1, HF_RELU = 2 };
/* Curvature matrix for hf_hvp / hf_cg / hf_bicgstab; hf_iterate also takes
 * HF_HYBRID (the Hybrid-CG policy of Sec. 3). */
enum { HF_HESSIAN = 0, HF_GAUSS_NEWTON = 1, HF_HYBRID = 2 };
/* Newton-system solver of hf_iterate. */
enum { HF_SOLVER_CG = 0, HF_SOLVER_BICGSTAB = 1 };
/* Arithmetic of the GEMMs (every other step is fp32, reductions fp64):
 *   HF_FP32         fp32 operands, fp32 MFMA, fp32 accumulation;
 *   HF_BF16_INPUTS  every GEMM operand (X, W, v, the activations and deltas
 *                   of the forward, backward, R-forward and R-backward
 *                   passes) rounded to bf16 (nearest even), bf16 MFMA with
 *                   fp32 accumulation; biases, epilogues (phi, phi', phi''),
 *                   the softmax and R-softmax rows, the phi'' cache, the
 *                   weight-gradient sums and all CG arithmetic stay fp32. */
enum { HF_FP32 = 0, HF_BF16_INPUTS = 1 };

enum {
  HF_OK = 0,
  HF_EINVAL = -1,     /* bad argument (null, misaligned, out of range)      */
  HF_ENOMEM = -2,     /* host allocation failed                            */
  HF_EHIP = -3,       /* a HIP runtime call failed                         */
  HF_ELABEL = -4,     /* a label outside [0, d_L) was seen (device check)  */
  HF_ENUMERIC = -5,   /* NaN or Inf in a CG scalar                         */
  HF_EWORKSPACE = -6  /* no workspace set, or it is too small              */
};

/* Limits checked by hf_create. */
#define HF_MAX_LAYERS 16
#define HF_MAX_CLASSES 4096

/*
 * hf_create: build a context for the network d_0-d_1-...-d_L.
 *   dims      host array of n_dims = L + 1 >= 2 positive sizes; d_L is the
 *             number of classes (<= HF_MAX_CLASSES); L <= HF_MAX_LAYERS.
 *   act       HF_SIGMOID | HF_TANH | HF_RELU for hidden layers.
 *   prec      HF_FP32 or HF_BF16_INPUTS.
 *   max_batch largest B any later call may use (>= 1); every B x d_l
 *             buffer and n must stay below 2^31 elements.
 *   hip_stream a hipStream_t for all device work of the context (NULL: the
 *             null stream); hf_set_stream changes it later.
 *   out       receives the context.  Returns HF_EINVAL on bad arguments.
 * No device call is made; the context holds no device memory.
 */
int hf_create(const int32_t* dims, int32_t n_dims, int32_t act, int32_t prec,
              int64_t max_batch, void* hip_stream, hf_ctx** out);

/* Free a context (host memory, events, pinned host staging).  NULL is ok. */
int hf_destroy(hf_ctx* ctx);

/* Stream (a hipStream_t) for all later device work; NULL = null stream. */
int hf_set_stream(hf_ctx* ctx, void* hip_stream);

/* n = sum_l d_l (d_{l-1} + 1), or -1 for a NULL context. */
int64_t hf_num_params(const hf_ctx* ctx);

/* Bytes of device workspace for calls of up to `batch` rows (batch <= 0:
 * max_batch).  0 for a NULL context or batch > max_batch.  Grows with
 * batch. */
size_t hf_workspace_bytes(const hf_ctx* ctx, int64_t batch);

/* Hand the context a device workspace, 256-byte aligned, of `bytes` bytes.
 * The context lays it out for the largest batch b <= max_batch with
 * hf_workspace_bytes(ctx, b) <= bytes; later calls with more than b rows
 * return HF_EWORKSPACE (as does a workspace too small for one row).  The
 * caller keeps ownership and must keep it alive while the context uses it,
 * and must not write to it meanwhile.  Contents need no initialisation: the
 * call clears what needs clearing (for HF_BF16_INPUTS, the operand padding)
 * and synchronises the device.  A new workspace discards the old one's
 * contents (such as the cache of a solve). */
int hf_set_workspace(hf_ctx* ctx, void* dev_ptr, size_t bytes);

/*
 * hf_loss_grad: f and g = grad f at theta = W on the batch (X, y) of B rows
 * (Alg. 1 step 1; the per-node gradient of Alg. 2).
 *   W     device, n fp32 (parameter layout above)
 *   X, y  device, B x d_0 fp32 and B int32
 *   loss  device, 1 fp32: f = (1/B) sum_i [logsumexp(z_i) - z_{i,y_i}]
 *   grad  device, n fp32
 * Asynchronous.  A label outside [0, d_L) raises a device flag reported as
 * HF_ELABEL by the next hf_check or hf_cg.
 */
int hf_loss_grad(hf_ctx* ctx, const float* W, const float* X,
                 const int32_t* y, int64_t B, float* loss, float* grad);

/*
 * hf_hvp: one curvature-vector product on the batch (X, y) of B rows,
 * without damping (Sec. 2.1, paragraph after Alg. 1; the per-node product of
 * Alg. 2):
 *   mode HF_HESSIAN      out = H v, exact Hessian of f by the R-operator
 *   mode HF_GAUSS_NEWTON out = G v = J^T H_L J v (labels unused; y may be NULL)
 *   v, out device, n fp32.  Asynchronous.
 */
int hf_hvp(hf_ctx* ctx, const float* W, const float* X, const int32_t* y,
           int64_t B, const float* v, int32_t mode, float* out);

/* Result of hf_cg (host struct). */
typedef struct hf_cg_info {
  int32_t iters;      /* completed updates of the iterate                   */
  int32_t products;   /* curvature products evaluated                       */
  int32_t neg_curv;   /* 1 if the solve stopped on p^T B_k p <= 0           */
  int32_t neg_iter;   /* CG iteration j of the detection, else -1           */
  double pBp;         /* p^T B_k p at the detection (kappa)                 */
  double pHp;         /* p^T A p = kappa - lambda ||p||^2 at the detection  */
  double gTd;         /* g^T d~ for the returned direction (<= 0)           */
  double rr0;         /* ||g||^2                                            */
  double rr_final;    /* ||r||^2 at exit                                    */
  int32_t status;     /* HF_OK, HF_ENUMERIC or HF_ELABEL                    */
  int32_t replayed;   /* 1 if the iterations were replayed from one captured
                         graph of an iteration (no kernel timing, kept
                         iterates or trace on the context), else 0          */
} hf_cg_info;

/*
 * hf_cg: CG-Minimize(B_k, -g) with B_k = A + lambda I, A = H or G on the
 * fixed curvature batch (Xc, yc) of Bc rows at theta = W (Alg. 1 steps 3-4;
 * Alg. 2 builds the operator from one minibatch).
 *   g          device, n fp32: the gradient (may come from a larger batch)
 *   damping    lambda >= 0
 *   max_iters  fixed iteration budget >= 0 (Sec. 2.2)
 *   rel_tol    stop when ||r||^2 <= rel_tol^2 ||g||^2; 0 disables
 *   step       device, n fp32: the iterate at exit; -g when negative
 *              curvature is met at the first iteration (Sec. 2.1)
 *   neg_dir    device, n fp32: d~ = -sgn(g^T p) p for the detected p
 *              (Sec. 2.2), zeros when there was no detection
 *   info       host struct, filled on return
 * Starts from x_0 = 0.  The loop runs on the device with device-resident
 * scalars; the call synchronises the stream before it returns.
 */
int hf_cg(hf_ctx* ctx, const float* W, const float* Xc, const int32_t* yc,
          int64_t Bc, const float* g, float damping, int32_t max_iters,
          float rel_tol, int32_t mode, float* step, float* neg_dir,
          hf_cg_info* info);

/*
 * hf_pcg: hf_cg preconditioned by the diagonal M (the pre-conditioning of
 * Martens' HF that Sec. 2.1 lists): z = M^-1 r, p_0 = -z_0,
 * alpha = r.z / p^T B_k p, beta = r'.z' / r.z, p = -z' + beta p.  The
 * detection test p^T B_k p <= 0, the returned step (-g at the first
 * iteration), the orientation of d~ and the relative stop on |r| / |g| are
 * those of hf_cg.
 *   minv   device, n fp32 (parameter layout), the diagonal of M^-1, > 0;
 *          e.g. (F + lambda)^(-3/4) with F from hf_fisher_diag
 * Other arguments, outputs and errors as for hf_cg.
 */
int hf_pcg(hf_ctx* ctx, const float* W, const float* Xc, const int32_t* yc,
           int64_t Bc, const float* g, float damping, int32_t max_iters,
           float rel_tol, int32_t mode, const float* minv, float* step,
           float* neg_dir, hf_cg_info* info);

/*
 * hf_fisher_diag: out = (1/B) sum_b grad l_b (.) grad l_b, the batch average
 * of the squared per-example gradients of the cross-entropy l_b of example
 * b (parameter layout; the diagonal Martens' preconditioner is built from).
 * One forward and one backward pass; the weight blocks are the weight-
 * gradient contraction of squared operands (HF_BF16_INPUTS: of the bf16
 * operands squared and rounded to bf16 again, accumulated in fp32).
 * X, y, B as for hf_loss_grad; out device, n fp32.  Asynchronous on the
 * context's stream.
 */
int hf_fisher_diag(hf_ctx* ctx, const float* W, const float* X,
                   const int32_t* y, int64_t B, float* out);

/*
 * hf_bicgstab: Bi-CG-STAB (Alg. 3; the solver behind the paper's results,
 * Sec. 2.1 footnote) for B_k d = -g with B_k = A + lambda I, A = H or G on
 * the fixed curvature batch (Xc, yc) of Bc rows at theta = W, from d = 0
 * with r0* = r0 (Alg. 2: "starting point 0").  Two curvature products per
 * iteration.  Every iterate x is a candidate direction (Sec. 2.2): its
 * curvature x^T A x (from x^T B x = -(g, x) - (r, x), r being the residual)
 * marks it Newton-type (> 0) or negative-curvature (< 0).
 *   step      device, n fp32: the final iterate (the Newton-system solution)
 *   neg_dir   device, n fp32: the FIRST negative-curvature candidate,
 *             oriented d~ = -sgn(g^T x) x, or zeros if none was met
 *   info      iters = completed iterations, products = curvature products,
 *             neg_curv / neg_iter = whether and at which iteration the first
 *             negative-curvature candidate appeared, pBp = d~^T B d~,
 *             pHp = d~^T A d~ (< 0), gTd = g^T d~ (< 0), rr0 = |g|^2,
 *             rr_final = |r|^2 at exit
 * The solve runs max_iters iterations unless the relative residual falls
 * below rel_tol (0 disables) or a denominator of the recurrences vanishes
 * ((A p, r0*) = 0 or (r, r0*) = 0; A s = 0 takes gamma = 0).  Arguments as
 * for hf_cg; the call synchronises the stream before it returns.
 */
int hf_bicgstab(hf_ctx* ctx, const float* W, const float* Xc, const int32_t* yc,
                int64_t Bc, const float* g, float damping, int32_t max_iters,
                float rel_tol, int32_t mode, float* step, float* neg_dir,
                hf_cg_info* info);

/*
 * hf_pbicgstab: hf_bicgstab preconditioned on the right by the diagonal M
 * (Martens' pre-conditioning, listed in Sec. 2.1, applied to Alg. 3; the
 * paper gives no preconditioned form, and right preconditioning is the one
 * that keeps the residual of the original system).  It is Bi-CG-STAB on
 * B_k M^-1 y = -g with d = M^-1 y: the two products of an iteration are
 * taken of M^-1 p and M^-1 s, and the iterate advances along them,
 * x += alpha M^-1 p + gamma M^-1 s.  r stays -g - B_k x, so the candidate
 * curvature, the breakdown tests and the relative stop on |r| / |g| are
 * those of hf_bicgstab.
 *   minv   device, n fp32 (parameter layout), the diagonal of M^-1, > 0
 * Other arguments, outputs and errors as for hf_bicgstab.
 */
int hf_pbicgstab(hf_ctx* ctx, const float* W, const float* Xc,
                 const int32_t* yc, int64_t Bc, const float* g, float damping,
                 int32_t max_iters, float rel_tol, int32_t mode,
                 const float* minv, float* step, float* neg_dir,
                 hf_cg_info* info);

/*
 * hf_loss: the objective alone, f = (1/B) sum_i [logsumexp(z_i) - z_{i,y_i}]
 * at theta = W on the batch (X, y) of B rows (the forward pass only; the
 * line search of Alg. 2 evaluates it at trial points).
 *   loss  device, 1 fp32.  Asynchronous; labels checked as in hf_loss_grad.
 */
int hf_loss(hf_ctx* ctx, const float* W, const float* X, const int32_t* y,
            int64_t B, float* loss);

/* Parameters of hf_iterate (host struct). */
typedef struct hf_iter_params {
  int32_t solver;         /* HF_SOLVER_CG or HF_SOLVER_BICGSTAB              */
  int32_t curvature;      /* HF_HESSIAN, HF_GAUSS_NEWTON or HF_HYBRID         */
  float damping;          /* lambda >= 0                                      */
  int32_t max_iters;      /* solver iteration budget >= 0 (Sec. 2.2)         */
  float rel_tol;          /* relative residual stop against |g|, 0 = off     */
  float eta;              /* warm start x0 = eta * delta; 0 starts from 0    */
  float armijo_c;         /* c of the Armijo condition, in (0, 1)            */
  float shrink;           /* step reduction per rejected trial, in (0, 1)    */
  int32_t max_backtracks; /* reductions tried per candidate, >= 0            */
  int32_t adapt_damping;  /* 1: compute rho and the next lambda (LM rule)   */
  int32_t keep_cap;       /* CG-backtracking: iterates kept, 0 = off        */
  float* keep_buf;        /* device, keep_cap * n fp32, caller-owned         */
  int32_t precondition;   /* 1: preconditioned solve, M = (F + lambda)^xi   */
  float precond_exp;      /* xi >= 0 (Martens: 3/4)                          */
} hf_iter_params;

/* Result of hf_iterate (host struct). */
typedef struct hf_iter_info {
  hf_cg_info solve;       /* the solve; products include the warm start's   */
  int32_t mode_used;      /* HF_HESSIAN or HF_GAUSS_NEWTON                    */
  int32_t direction;      /* 0 the solver's step, 1 the negative-curvature
                             direction, -1 no candidate accepted            */
  int32_t accepted;       /* 1 if a step satisfied the Armijo condition      */
  int32_t evals;          /* objective evaluations in the line searches      */
  double f0, f1;          /* f before and after (f1 = f0 if none accepted)   */
  double alpha;           /* accepted step length, 0 if none                */
  double gTd;             /* g^T delta for the chosen direction             */
  int32_t backtrack_iter; /* solver iterate chosen by backtracking, -1 off  */
  double rho;             /* reduction ratio (-inf: undefined; nan: off)    */
  double damping_next;    /* lambda for the next iteration                  */
} hf_iter_info;

/*
 * hf_iterate: one iteration of the distributed HF method on one worker's
 * share (Alg. 2, one k; Alg. 1):
 *   1. f and g at theta = W on the batch (X, y) of B rows;
 *   2. the curvature on the batch (Xc, yc) of Bc rows: H, G, or HF_HYBRID:
 *      H, except in the iteration right after a Hessian solve that met
 *      negative curvature, which uses G (Sec. 3); *hybrid_state carries
 *      this between calls (in/out, 0 initially; ignored otherwise);
 *   3. the Newton system (A + lambda I) d = -g by CG-Minimize (Alg. 1) or
 *      Bi-CG-STAB (Alg. 3), from 0 or from eta * delta (Alg. 2);
 *   4. the candidate directions (Sec. 2.2): the solver's step if
 *      g^T step < 0, and the oriented negative-curvature direction if one
 *      was met, rescaled to the step's length (to |g| if the step is 0);
 *   5. for each candidate, Armijo backtracking (Alg. 2): alpha = 1, then
 *      alpha *= shrink until f(W + alpha d) <= f + c alpha g^T d, at most
 *      max_backtracks reductions; the candidate reaching the lower f wins;
 *   6. W += alpha d in place, and delta = d (zeros if none was accepted).
 * CG-backtracking (keep_cap > 0; Sec. 2.2 takes the solver's iterates as
 * candidates for it, after Martens 2010): the solver keeps its iterate after
 * j updates for j = 1, then j <- max(j + 1, ceil(13 j / 10)), j < max_iters,
 * the latest keep_cap of them, in keep_buf (keep_cap consecutive vectors of
 * n floats, overwritten).  f is then evaluated from the final iterate
 * backwards while it decreases; the last iterate before it rises replaces
 * the solver's step in 4., and its f serves as the Armijo trial at
 * alpha = 1.  Damping (adapt_damping = 1; Alg. 1 adjusts lambda in its
 * second step): rho = (f1 - f0) / (m(p) - m(0)) for the accepted update
 * p = alpha d, with m the damped quadratic model of eq. (1) and B p from one
 * stateless curvature product at the old W; damping_next = 3/2 lambda if
 * rho < 1/4 (also when nothing was accepted or m(p) >= m(0), reported as
 * rho = -inf), 2/3 lambda if rho > 3/4, else lambda.  Without it rho is NaN
 * and damping_next = damping.  Preconditioning (precondition = 1;
 * damping > 0 only): the gradient pass of 1. also forms F as hf_fisher_diag
 * does on (X, y), and the solve of 3. is hf_pcg or hf_pbicgstab with
 * M^-1 = (F + lambda)^(-xi).
 *   W      device, n fp32, in/out.  X, y / Xc, yc as for hf_loss_grad /
 *          hf_cg (yc may be NULL only for HF_GAUSS_NEWTON).
 *   delta  device, n fp32, in/out: delta_{k-1} in, delta_k out.
 * The objective values that decide the line search are reduced in fp64.
 * Synchronises the stream; uses the workspace's solver vectors.
 */
int hf_iterate(hf_ctx* ctx, float* W, const float* X, const int32_t* y,
               int64_t B, const float* Xc, const int32_t* yc, int64_t Bc,
               const hf_iter_params* params, int32_t* hybrid_state,
               float* delta, hf_iter_info* info);

/*
 * hf_set_trace: lock-step diagnostic of the solvers' curvature products.
 * Every later solve on ctx (hf_cg, hf_pcg, hf_bicgstab, hf_pbicgstab and
 * the solve inside hf_iterate) copies the operand v (for hf_pbicgstab
 * M^-1 p and M^-1 s) and the undamped result A v of each of its first
 * `cap` curvature products k into buf: slot 2k (n floats at
 * buf + 2k n) gets v, slot 2k + 1 gets A v (A = H or G of the solve, on its
 * cached curvature batch; the product B_k v of Alg. 1 step 3 is A v +
 * lambda v).  Products are numbered in the order the solve evaluates them:
 * a warm start's product is k = 0; CG's iteration j is k = j (+1 after a
 * warm start); Bi-CG-STAB's iteration j is k = 2j (on p) and 2j + 1 (on s).
 * Slots of products the solve did not evaluate are left untouched.
 *   buf  device, 2 cap n fp32, 16-byte aligned, caller-owned; it must stay
 *        alive while tracing is on.  cap = 0 (buf ignored) turns it off.
 * Returns HF_EINVAL for cap < 0 or a NULL / misaligned buffer with cap > 0.
 * Costs two vector copies per traced product.
 */
int hf_set_trace(hf_ctx* ctx, float* buf, int32_t cap);

/* SHA-256 (hex) of the sources the library was built from. */
const char* hf_build_id(void);

/* Bytes of the device scratch that hf_hvp_noalloc uses in place of a
 * workspace: one array per GPU, held until the process ends. */
#define HF_NOALLOC_SCRATCH_BYTES ((size_t)128 << 20)

/*
 * hf_hvp_noalloc: hf_hvp for callers that cannot allocate device memory or
 * hand over a workspace (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation).  It computes what hf_hvp computes, but
 * its scratch is a static device array of HF_NOALLOC_SCRATCH_BYTES per GPU
 * instead of the context's workspace (none needs to be set).  It makes no
 * allocating call (no hipMalloc, hipFree, memset node or host-side device
 * allocation), is asynchronous on the context's stream, and can be captured
 * into a graph.  It always runs the kernels that fuse the two forward and the
 * two backward passes.  So does hf_hvp, with the same bits, except where the
 * passes of a solve serve a shape better (fp32: fewer than 128 tiles of
 * 128 x 128 in the first layer; bf16: at least 256 of 256 x 256); there the
 * two differ by the rounding of sums taken in another order.
 *   label_err  device int32 or NULL: set to 0 by the call, then to 1 if a
 *              label outside [0, d_L) was seen (hf_hvp reports this through
 *              hf_check instead; without label_err it is not reported).
 * The scratch holds the activations, deltas and split-K partials of one
 * product at B rows (less than hf_workspace_bytes(ctx, B), which also
 * holds the solvers' vectors); a batch whose layout needs more than
 * HF_NOALLOC_SCRATCH_BYTES returns HF_EWORKSPACE before any device work.
 * Every call on one GPU shares that GPU's scratch and leaves its contents
 * there: calls that may overlap on one GPU (other streams, other threads,
 * other contexts) race and must be serialised by the caller.
 * The context's workspace, if any, is not touched.  Other arguments and
 * errors as for hf_hvp; the context's kernel profiler does not time it.
 */
int hf_hvp_noalloc(hf_ctx* ctx, const float* W, const float* X,
                   const int32_t* y, int64_t B, const float* v, int32_t mode,
                   float* out, int32_t* label_err);

/* Synchronise the stream and report a device-detected error (HF_ELABEL)
 * raised since the last hf_check; clears the flag. */
int hf_check(hf_ctx* ctx);

/* Message for the last failed call on ctx ("" if none); static text for a
 * NULL context. */
const char* hf_last_error(const hf_ctx* ctx);

/* Static name of an HF_* code. */
const char* hf_strerror(int32_t code);

/*
 * Kernel timing.  When enabled, every kernel launch carries a start/stop HIP
 * event pair bound to its dispatch on the context's stream, and its
 * algorithmic work (flops for the contractions, bytes for memory-bound
 * kernels) is accumulated per kernel name.  hf_prof_get synchronises the
 * stream.  hf_prof_only restricts the events to the launches of one kernel
 * name (NULL or "": every kernel; HF_EINVAL while timing is off) until it
 * is called again or timing is turned off (hf_prof_reset keeps it);
 * launches and work are still counted for every name, the others' times
 * stay 0.
 * Events cost time of their own (a few microseconds per launch), which
 * matters for small kernels.
 */
int hf_prof_enable(hf_ctx* ctx, int32_t on);
int hf_prof_only(hf_ctx* ctx, const char* name);
int hf_prof_reset(hf_ctx* ctx);
int32_t hf_prof_count(hf_ctx* ctx);
int hf_prof_get(hf_ctx* ctx, int32_t i, const char** name, int64_t* launches,
                double* total_ms, double* flops, double* bytes);

/*
 * ------------------------------------------------------------------------
 * The vocabulary ends of a token model: the embedding in front of a net, and
 * behind it the softmax head over a vocabulary larger than HF_MAX_CLASSES,
 * with the loss of hard labels or of a teacher's top logits.  With tied
 * weights the embedding and the head share one matrix and one gradient.  What
 * lies between them (rows in, their gradient back) is the caller's, or made of
 * hf_gated's below: an hf_ctx takes no rows from an embedding that is trained
 * with it, and gives no activations to a head; and the solvers have no curvature
 * product of these.
 *
 * A context (hf_vocab) holds the vocabulary V, the width D and the type of
 * the rows, the matrices and their gradients: fp32 or bf16 (sums, softmax
 * statistics and losses are fp32, the sum over the rows fp64; each output is
 * rounded to its type once).  Matrices are row-major; rows may lie `ld`
 * elements apart and start at any element (rows of 16-byte multiples and
 * widths that are multiples of 64 are read in place, others are packed in
 * the workspace first).
 * Labels, tokens and ids are int32 in [0, V), or HF_IGNORE where a place is
 * masked; any other value counts as masked and raises HF_ELABEL in the next
 * hf_vocab_check.  Rows without a target count nothing: no loss, a zero row
 * of dX, nothing in dW, whatever X holds there.
 * Outputs may not overlap inputs.
 * Memory, streams and errors as for hf_ctx: device pointers owned by the
 * caller, one caller-provided workspace, everything asynchronous on the
 * context's stream, HF_* codes.  Calls make no allocation and can be captured
 * into a graph.  As they share the workspace, a call waits for the context's
 * calls before it, whatever streams they are on: hf_vocab_set_stream orders the
 * new stream behind the old one (which must still exist), or, while one of the
 * two is captured, the next call does (until then the stream of the calls
 * before it must exist; while that one is captured, the call is refused).
 * Captured calls, and graphs that share a workspace, are the caller's to order.
 * The current device must be the stream's.  Repeated calls give the same bits,
 * whatever the workspace's size.
 */
typedef struct hf_vocab hf_vocab;

enum { HF_TYPE_FP32 = 0, HF_TYPE_BF16 = 1 };
/* A masked label, token or id. */
#define HF_IGNORE (-100)
/* Limits: vocabulary, width, rows per call, teacher logits per row. */
#define HF_VOCAB_MAX (1 << 22)
#define HF_VOCAB_MAX_WIDTH 65536
#define HF_VOCAB_MAX_ROWS 262144
#define HF_VOCAB_MAX_TOP 128

/* Build a context for calls of up to max_rows rows; HF_EINVAL outside the
 * limits.  No device call is made. */
int hf_vocab_create(int64_t vocab, int32_t width, int32_t type,
                    int64_t max_rows, void* hip_stream, hf_vocab** out);
/* Free a context.  NULL is ok. */
int hf_vocab_destroy(hf_vocab* ctx);
/* Stream (a hipStream_t) of later calls, after an error as well; NULL = null
 * stream. */
int hf_vocab_set_stream(hf_vocab* ctx, void* hip_stream);
/* Bytes of workspace for calls of up to `rows` rows (<= 0: max_rows); 0 for a
 * NULL context or rows > max_rows.  Grows with rows. */
size_t hf_vocab_workspace_bytes(const hf_vocab* ctx, int64_t rows);
/* Hand over a device workspace, 256-byte aligned; calls with more rows than
 * its bytes serve return HF_EWORKSPACE.  Synchronises the device. */
int hf_vocab_set_workspace(hf_vocab* ctx, void* dev_ptr, size_t bytes);

/*
 * hf_vocab_loss: softmax cross entropy of the logits z = X W^T,
 *   l_i = logsumexp(z_i) - z_{i, y_i},  loss = sum_i l_i / denom
 * in tiles of the vocabulary: the logits are never stored.
 *   X         rows x D, ldx >= D elements apart
 *   W         V x D, ldw apart
 *   y         rows labels
 *   denom     divides the sum; 0: the number of counted rows (loss 0 if none)
 *   loss      1 fp32
 *   row_loss  rows fp32 (0 where a row does not count), or NULL
 */
int hf_vocab_loss(hf_vocab* ctx, const void* X, int64_t ldx, const void* W,
                  int64_t ldw, const int32_t* y, int64_t rows, float denom,
                  float* loss, float* row_loss);

/*
 * hf_vocab_loss_grad: hf_vocab_loss and its gradients
 *   dX = delta W (rows x D),  dW = delta^T X (V x D),
 *   delta = (softmax(z) - e_y) / denom.
 * The workspace keeps a call's logits: all of up to 128 rows, whatever the
 * vocabulary (of a word, 4 bytes a row, the rows up to a multiple of 64; with
 * bf16 8, up to a multiple of 32); of more rows at most 1.5 GiB (fp32; with
 * bf16 exponentials in fp16: softmax(z) to 2^-12 of itself, or to 2^-40 of the
 * largest among up to 128 neighbours), the whole ones or a piece of the
 * vocabulary's, the others being computed again piece by piece.  delta is
 * rounded to the type (bf16 calls of up to 128 rows: to two terms of it) for the
 * two products.
 *   dX, dW      either may be NULL (not both): not computed
 *   accumulate  1: dW += instead of dW = (with tied weights, or over
 *               minibatches); dX is always written whole
 */
int hf_vocab_loss_grad(hf_vocab* ctx, const void* X, int64_t ldx,
                       const void* W, int64_t ldw, const int32_t* y,
                       int64_t rows, float denom, float* loss, float* row_loss,
                       void* dX, int64_t lddx, void* dW, int64_t lddw,
                       int32_t accumulate);

/*
 * hf_vocab_distill: divergence from a teacher known by the top logits of each
 * row, at temperature tau:
 *   q_i = softmax(t_i / tau) over the row's list,  p_i = softmax(z_i / tau)
 *   over the vocabulary,
 *   l_i = tau^2 sum over the listed ids v of q_iv (log q_iv - log p_iv)
 *   ids  rows x top ids, ldi apart; HF_IGNORE where the list has ended
 *   t    rows x top fp32 teacher logits, ldt apart; -inf counts as masked
 *   top  1 .. HF_VOCAB_MAX_TOP;  tau in [1e-4, 1e4]
 * An id that a row lists twice has the sum of its probabilities as q_iv.
 * Few rows' logits are stored in the workspace where that is quicker.
 * Other arguments as for hf_vocab_loss.
 */
int hf_vocab_distill(hf_vocab* ctx, const void* X, int64_t ldx, const void* W,
                     int64_t ldw, const int32_t* ids, int64_t ldi,
                     const float* t, int64_t ldt, int32_t top, float tau,
                     int64_t rows, float denom, float* loss, float* row_loss);

/* hf_vocab_distill_grad: hf_vocab_distill and its gradients, those of
 * hf_vocab_loss_grad with delta = tau (p - q) / denom. */
int hf_vocab_distill_grad(hf_vocab* ctx, const void* X, int64_t ldx,
                          const void* W, int64_t ldw, const int32_t* ids,
                          int64_t ldi, const float* t, int64_t ldt,
                          int32_t top, float tau, int64_t rows, float denom,
                          float* loss, float* row_loss, void* dX, int64_t lddx,
                          void* dW, int64_t lddw, int32_t accumulate);

/* hf_vocab_embed: out_i = scale E[tok_i] (rows x D, ldo apart), zeros where
 * tok_i is masked.  E is V x D, lde apart; scale finite. */
int hf_vocab_embed(hf_vocab* ctx, const void* E, int64_t lde,
                   const int32_t* tok, int64_t rows, float scale, void* out,
                   int64_t ldo);

/* hf_vocab_embed_grad: its gradient, dE_v = scale sum_{i: tok_i = v} dout_i
 * (V x D, lde apart), summed in fp32 in a fixed order; rows of dE without a
 * token are zero.  accumulate = 1: dE += instead (rows without a token are
 * left as they are). */
int hf_vocab_embed_grad(hf_vocab* ctx, const int32_t* tok, int64_t rows,
                        float scale, const void* dout, int64_t ldd, void* dE,
                        int64_t lde, int32_t accumulate);

/* Synchronise the stream and report HF_ELABEL raised since the last check;
 * clears the flag. */
int hf_vocab_check(hf_vocab* ctx);
/* Message for the last failed call on ctx. */
const char* hf_vocab_last_error(const hf_vocab* ctx);

/*
 * ------------------------------------------------------------------------
 * The gated feed-forward block of a token model, which lies between its two
 * ends: with D the width and F the hidden width,
 *   g = X Wg^T,  u = X Wu^T,  h = phi(g) u,  Y = h Wd^T
 *   X, Y  rows x D;  Wg, Wu  F x D;  Wd  D x F
 * in training, with what the gradient needs kept in full or in 8 bits, and in
 * serving, down to one token, with the matrices as they are or in 8-bit codes.
 *
 * A context (hf_gated) holds D, F, the activation phi and the type of the
 * rows, the matrices and their gradients: fp32 or bf16 (sums and the activation
 * are fp32; h, and in the gradient dg and du, are rounded to the type for the
 * product that reads them, with bf16 calls of up to 128 rows to two terms of it,
 * or not at all; each output is rounded to its type once).  Matrices are row-major; rows may lie `ld` elements
 * apart and start at any element (forward calls of up to 64 rows read them in
 * place, but for bf16 ones of more than 32 with long rows of Wd; others rows of
 * 16-byte multiples and widths that are multiples of 64, of codes 128; what lies
 * otherwise is copied to the workspace first).  Columns and rows around an
 * output are left as they were.  Outputs may not overlap inputs.
 * Memory, streams, the order of calls and errors as for hf_vocab; calls make no
 * allocation and can be captured into a graph.  hf_gated_pack, _unpack and
 * _codes use no workspace, but keep the order of calls.  Repeated calls give the
 * same bits (operands that lie otherwise may be summed in another order).  Rows
 * do not mix: a row with a number that is not finite spoils its own results and
 * the matrices' gradients.
 */
typedef struct hf_gated hf_gated;

/* Activations, besides HF_SIGMOID, HF_TANH and HF_RELU: z sigmoid(z);
 * z Phi(z); and z Phi(z) with Phi(z) = (1 + tanh(sqrt(2 / pi) (z + 0.044715
 * z^3))) / 2. */
enum { HF_SILU = 3, HF_GELU = 4, HF_GELU_TANH = 5 };
/* What hf_gated_forward keeps of g and u. */
enum { HF_KEEP_NONE = 0, HF_KEEP_FULL = 1, HF_KEEP_CODES = 2 };
/* Limits: width, hidden width and columns of an array; rows per call; rows of
 * a matrix that is turned into codes, and channels of a product. */
#define HF_GATED_MAX_WIDTH 65536
#define HF_GATED_MAX_ROWS 262144
#define HF_GATED_MAX_OUT (1 << 22)
/* Neighbours in a row that share a scale in a checkpoint. */
#define HF_CODE_BLOCK 32

/* Build a context for calls of up to max_rows rows; HF_EINVAL outside the
 * limits.  No device call is made. */
int hf_gated_create(int32_t width, int32_t hidden, int32_t act, int32_t type,
                    int64_t max_rows, void* hip_stream, hf_gated** out);
/* Free a context.  NULL is ok. */
int hf_gated_destroy(hf_gated* ctx);
/* Stream (a hipStream_t) of later calls, after an error as well; NULL = null
 * stream. */
int hf_gated_set_stream(hf_gated* ctx, void* hip_stream);
/* Bytes of workspace for calls of up to `rows` rows (<= 0: max_rows); 0 for a
 * NULL context or rows > max_rows.  Grows with rows. */
size_t hf_gated_workspace_bytes(const hf_gated* ctx, int64_t rows);
/* Hand over a device workspace, 256-byte aligned; calls with more rows than
 * its bytes serve return HF_EWORKSPACE.  Synchronises the device. */
int hf_gated_set_workspace(hf_gated* ctx, void* dev_ptr, size_t bytes);

/*
 * hf_gated_forward: Y of the block, and what its gradient needs.
 *   X       rows x D, ldx >= D elements apart;  Y  rows x D, ldy apart
 *   Wg, Wu  F x D, ldg and ldu apart;  Wd  D x F, ldd apart
 *   keep    HF_KEEP_NONE; HF_KEEP_FULL: g and u in the type; HF_KEEP_CODES: in
 *           8 bits, as hf_gated_pack writes them (of the fp32 sums)
 *   kept    rows x 2 F, ldk apart: a row of g and then of u, in the type or as
 *           codes; ignored with HF_KEEP_NONE
 *   scale   HF_KEEP_CODES: rows x 2 ceil(F / 32) scale bytes, lds apart: g's
 *           and then u's
 */
int hf_gated_forward(hf_gated* ctx, const void* X, int64_t ldx, const void* Wg,
                     int64_t ldg, const void* Wu, int64_t ldu, const void* Wd,
                     int64_t ldd, int64_t rows, void* Y, int64_t ldy,
                     int32_t keep, void* kept, int64_t ldk, uint8_t* scale,
                     int64_t lds);

/*
 * hf_gated_grad: the block's gradients from that of Y and what was kept,
 *   dh = dY Wd,  du = dh phi(g),  dg = dh u phi'(g)
 *   dX = dg Wg + du Wu,  dWg = dg^T X,  dWu = du^T X,  dWd = dY^T h
 * relu's slope at 0 is 0.
 *   X, xscale   X as forward had it (xscale NULL), or its codes and scale bytes
 *               from hf_gated_pack (ldx and ldxs apart): read for dWg and dWu
 *   keep, kept, scale   what hf_gated_forward has kept
 *   dX, dWg, dWu, dWd   shaped like X and the matrices, each or NULL (not all):
 *               not computed
 *   accumulate  1: dWg, dWu and dWd += instead of = (over minibatches); dX is
 *               always written whole
 */
int hf_gated_grad(hf_gated* ctx, const void* X, int64_t ldx,
                  const uint8_t* xscale, int64_t ldxs, const void* Wg,
                  int64_t ldg, const void* Wu, int64_t ldu, const void* Wd,
                  int64_t ldd, int32_t keep, const void* kept, int64_t ldk,
                  const uint8_t* scale, int64_t lds, const void* dY,
                  int64_t lddy, int64_t rows, void* dX, int64_t lddx, void* dWg,
                  int64_t lddg, void* dWu, int64_t lddu, void* dWd,
                  int64_t lddd, int32_t accumulate);

/*
 * hf_gated_pack: a checkpoint of rows x cols numbers of the type in 8 bits.
 * HF_CODE_BLOCK neighbours of a row (the last block of a row may be shorter)
 * share a scale byte b, and a number's code q in [-127, 127] stands for
 * q 2^(b - 127):
 *   b = 127 + e - 6, 2^e the largest power of two up to the block's largest
 *   magnitude, one more where that one's code would round to 128; at least 0
 *   q = the number over 2^(b - 127), rounded to nearest, ties to even
 * Each number is within half a step 2^(b - 127), at most 2^-6.99 of the
 * block's largest.  A block with a NaN or an infinity has b = 255 and unpacks to
 * NaN.  hf_gated_unpack writes the numbers in the type: exactly, as 7 bits and a
 * power of two (below bf16's smallest normal number, rounded; 64 2^122, next to
 * the types' largest number, is past it: infinity).
 *   codes  rows x cols, ldc apart;  scale  rows x ceil(cols / 32), lds apart
 */
int hf_gated_pack(hf_gated* ctx, const void* X, int64_t ldx, int64_t rows,
                  int64_t cols, int8_t* codes, int64_t ldc, uint8_t* scale,
                  int64_t lds);
int hf_gated_unpack(hf_gated* ctx, const int8_t* codes, int64_t ldc,
                    const uint8_t* scale, int64_t lds, int64_t rows,
                    int64_t cols, void* X, int64_t ldx);

/*
 * hf_gated_codes: rows of the type as 8-bit codes with a scale for each row (a
 * token's, or a matrix's channel's): s = max |x| / 127 in fp32, q = x / s
 * rounded to nearest, ties to even, in [-127, 127] (past which x / s may lie where
 * s is below fp32's normal numbers).  A row whose s is 0 (of zeros, or of numbers
 * below 2^-143) has codes 0; one with a NaN or an infinity has s = NaN and codes
 * 0.
 *   X  rows x cols;  codes  rows x cols, ldc apart;  scale  rows fp32
 */
int hf_gated_codes(hf_gated* ctx, const void* X, int64_t ldx, int64_t rows,
                   int64_t cols, int8_t* codes, int64_t ldc, float* scale);

/*
 * hf_gated_product: the product of two matrices of codes, y_tn = sa_t sb_n
 * sum_k A_tk B_nk, the sum exact in 32 bits, then rounded to fp32 and scaled by
 * one scale after the other, wherever in the type's range y is.
 *   A  rows x k codes, lda apart, with sa: rows fp32 scales
 *   B  n x k codes, ldb apart, with sb: n fp32 scales
 *   n  1 .. HF_GATED_MAX_OUT;  k  1 .. the larger of the context's widths
 *   Y  rows x n of the type, ldy apart
 */
int hf_gated_product(hf_gated* ctx, const int8_t* A, int64_t lda,
                     const float* sa, const int8_t* B, int64_t ldb,
                     const float* sb, int64_t rows, int64_t n, int64_t k,
                     void* Y, int64_t ldy);

/*
 * hf_gated_forward_codes: hf_gated_forward with the matrices as codes of
 * hf_gated_codes (F, F and D scales).  X's rows, and h's (of fp32), are turned
 * into codes on the way; every product is hf_gated_product's.
 */
int hf_gated_forward_codes(hf_gated* ctx, const void* X, int64_t ldx,
                           const int8_t* Wg, int64_t ldg, const float* sg,
                           const int8_t* Wu, int64_t ldu, const float* su,
                           const int8_t* Wd, int64_t ldd, const float* sd,
                           int64_t rows, void* Y, int64_t ldy);

/* Message for the last failed call on ctx. */
const char* hf_gated_last_error(const hf_gated* ctx);

#ifdef __cplusplus
}
#endif
#endif /* HF_H */
