/*
 * ls.h -- C ABI of the local-update SGD library for one NVIDIA B200 (sm_100a).
 *
 * The library runs the data-parallel hot path of periodic-averaging SGD
 * (PASGD, Section 2 of "Adaptive Communication Strategies to Achieve the Best
 * Error-Runtime Trade-off in Local-Update SGD") for m model replicas that all
 * live in one GPU's memory, and the AdaComm communication-period rule
 * (Section 4.2).  Every arithmetic step runs in CUDA kernels of this library;
 * there is no CPU fallback.
 *
 * Conventions
 *  - Every function returns an int status: LS_OK (0) or a negative LS_ERR_*.
 *    Nothing throws or aborts across this boundary.  ls_strerror() names a code.
 *  - "dev" pointers are CUDA device pointers on the current device, "host"
 *    pointers are ordinary host memory.  The library allocates no device
 *    memory: the caller allocates one state block of ls_state_bytes() bytes
 *    (256-byte aligned) and lends it to the handle until ls_destroy().
 *  - Kernels are enqueued on the CUDA stream given to ls_create() and the call
 *    returns without waiting unless stated otherwise.  An asynchronous CUDA
 *    error surfaces as LS_ERR_CUDA from a later call or from ls_sync().
 *  - A handle is not thread-safe.
 *
 * Model: a fully connected network
 *      x -> W_L relu( ... relu(W_1 x + b_1) ... ) + b_L
 *  with dims = (d_in, h_1, ..., d_out).  n_layers == 1 is a linear model
 *  (softmax regression, or least squares with LS_LOSS_MSE_HALF and d_out == 1).
 *
 * Flat parameter layout of one replica (P = ls_param_count() floats): for
 *  l = 1..L the matrix W_l as [dims[l]][dims[l-1]] row-major, then b_l
 *  (dims[l] floats) when has_bias.  Momentum buffers use the same layout.
 *  Inside the state block replica i's vector starts at i * ls_param_stride()
 *  floats (the stride is P rounded up to a multiple of 64 floats).
 */
#ifndef LS_H_
#define LS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LS_MAX_LAYERS 8
#define LS_MAX_REPLICAS 64
#define LS_MAX_BATCH 1024
#define LS_MAX_OUT 1024          /* largest d_out (width of the loss layer) */

enum {
  LS_OK = 0,
  LS_ERR_INVALID_ARG = -1,       /* null pointer, size out of range, bad enum, non-finite number */
  LS_ERR_BAD_HANDLE = -2,
  LS_ERR_STATE_SIZE = -3,        /* state block too small or misaligned */
  LS_ERR_NO_DATASET = -4,        /* ls_bind_dataset() has not been called */
  LS_ERR_ROW_RANGE = -5,         /* a mini-batch would read past the bound dataset */
  LS_ERR_CUDA = -6,              /* a CUDA runtime call failed; ls_last_cuda_error() has its code */
  LS_ERR_UNSUPPORTED = -7,       /* valid request that the library does not implement (e.g. weight decay) */
  LS_ERR_OVERFLOW = -8,          /* a result does not fit its type */
  LS_ERR_DEVICE_TIMEOUT = -9,    /* a bounded wait inside a kernel ran out; results of that launch are invalid */
  LS_ERR_TOO_LARGE = -10,        /* a size exceeds a fixed capacity of the entry point */
  LS_ERR_EXCHANGE = -11          /* the exchange callback of ls_set_shard() reported a failure */
};

enum { LS_LOSS_SOFTMAX_CE = 0, LS_LOSS_MSE_HALF = 1 };
enum { LS_GEMM_FP32 = 0, LS_GEMM_BF16 = 1 };
/* Element type of the tensors of the operators on raw buffers (ls_layer_norm, ls_vocab_loss, ls_orthogonalize, ...). */
enum { LS_DTYPE_FP32 = 0, LS_DTYPE_BF16 = 1 };
/* What an averaging step does with the per-replica momentum buffers.
 * AVERAGE: replaced by their mean like the parameters (makes tau = 1 equal to
 *          synchronous momentum SGD on the m-fold batch).
 * KEEP:    left alone (the independent-buffer scheme of Section 5.3).
 * RESET:   cleared (the local half of the block-momentum scheme, Section 5.3).
 * BLOCK:   block momentum (Section 5.3): local buffers cleared, and the averaging step
 *          applies a global momentum buffer u to the period's accumulated step:
 *            u_j = beta_glob u_{j-1} + G_j,   x_{(j+1)tau+1} = x_{j tau+1} - eta u_j,
 *          with x_{j tau+1} the synchronized model the period started from and
 *          G_j = (x_{j tau+1} - mean_i x^(i)) / eta the averaged displacement in gradient units
 *          (the sum of the averaged gradients when the local steps are plain SGD).
 *          beta_glob is spec.block_momentum; see ls_average for the exact arithmetic. */
enum { LS_MOMENTUM_AVERAGE = 0, LS_MOMENTUM_KEEP = 1, LS_MOMENTUM_RESET = 2, LS_MOMENTUM_BLOCK = 3 };

typedef struct ls_model_spec {
  int32_t n_layers;                  /* L, 1..LS_MAX_LAYERS */
  int32_t dims[LS_MAX_LAYERS + 1];   /* dims[0..L] */
  int32_t loss;                      /* LS_LOSS_* */
  int32_t has_bias;                  /* 0 or 1 */
  int32_t gemm_dtype;                /* LS_GEMM_*: input type of the matrix products (accumulation is fp32) */
  int32_t momentum_mode;             /* LS_MOMENTUM_* */
  float weight_decay;                /* must be 0 */
  float block_momentum;              /* beta_glob of Section 5.3, 0 <= beta < 1; read only in LS_MOMENTUM_BLOCK */
} ls_model_spec;

typedef struct ls_handle ls_handle;

const char* ls_strerror(int code);

/* ---- sizes ------------------------------------------------------------- */

/* P, the number of parameters of one replica.  (x in R^d of Section 2.) */
int ls_param_count(const ls_model_spec* spec, int64_t* P);

/* Housekeeping (no passage of the paper): bytes of the caller-allocated state block for m replicas and
 * mini-batches of `batch` rows: parameters, momentum, bf16 weight copies (bf16 models),
 * activation / gradient workspace, staging for host batches. */
int ls_state_bytes(int m, const ls_model_spec* spec, int batch, size_t* bytes);

/* ---- life cycle -------------------------------------------------------- */

/* Create a handle for m replicas (1..LS_MAX_REPLICAS) that train with
 * learning rate lr (eta of Section 2) and momentum factor `momentum`
 * (0 <= momentum < 1; 0 means plain SGD and the buffers are never touched).
 * state_dev: device block of >= ls_state_bytes() bytes, 256-byte aligned; it is
 * borrowed until ls_destroy().  All parameters and momentum buffers start at
 * zero (enqueued on `cuda_stream`, a cudaStream_t passed as void*, may be 0).
 * Creates one auxiliary CUDA stream and a few events; allocates a small pinned
 * host buffer; no device memory. */
int ls_create(ls_handle** h, int m, const ls_model_spec* spec, float lr, float momentum, int batch,
              void* state_dev, size_t state_bytes, void* cuda_stream);
int ls_destroy(ls_handle* h);
/* Wait for everything enqueued so far; returns LS_ERR_CUDA if any of it failed.
 * Every wait inside the kernels (on a barrier, on a copy) is bounded; one that runs out makes its kernel
 * record a code in the state block and return.  ls_sync() and every call that waits for the stream itself
 * (ls_eval_loss, ls_local_steps_host, the decision points of ls_run / ls_run_refined / ls_run_timed, the state
 * accessors) then return LS_ERR_DEVICE_TIMEOUT once and clear the record: the results of the launches since the
 * last successful wait are invalid (restore the replicas with ls_set_state), the handle itself stays usable. */
int ls_sync(ls_handle* h);
/* Housekeeping (no passage of the paper): exercises the report path above without touching any other kernel.
 * Enqueues a one-thread kernel that waits, for at most limit_cycles SM clock ticks (1 .. 2e9), on a barrier on
 * which nothing ever arrives, gives up, and records the failure like a training kernel would.  The next
 * ls_sync() returns LS_ERR_DEVICE_TIMEOUT, the one after it LS_OK.  Nothing faults or hangs: the wait is the
 * bounded one the library uses everywhere. */
int ls_selftest_wait_timeout(ls_handle* h, int64_t limit_cycles);
int ls_last_cuda_error(const ls_handle* h);
int ls_set_lr(ls_handle* h, float lr);

/* ---- replica state  (X_k = [x^(1) ... x^(m)] of the proof's notation) --- */

/* All workers start at the same point x_1 (Section 2): copy the P host floats
 * to every replica, clear every momentum buffer.  Synchronous. */
int ls_set_params(ls_handle* h, const float* x1_host);
/* Overwrite / read one replica's parameters and momentum (P host floats each;
 * either pointer may be NULL to skip it).  Synchronous. */
int ls_set_state(ls_handle* h, int replica, const float* params_host, const float* momentum_host);
int ls_get_state(ls_handle* h, int replica, float* params_host, float* momentum_host);
/* Device views of the packed replicas: base pointers and the stride between
 * replicas in floats.  The memory belongs to the state block.  Views are for
 * reading: the handle does not see a write through them (the bf16 copies that the
 * products of a bf16 model read, and the copy of the synchronized model that the
 * first local step after ls_set_params or an averaging step reads, keep the old
 * values).  Inside a replica, tensors start at multiples of 64 floats, and a bf16
 * model keeps the matrices of its wide layers in 32 x 32 blocks, not row-major. */
int ls_state_view(ls_handle* h, float** params_dev, float** momentum_dev, int64_t* stride_floats);

/* ---- data -------------------------------------------------------------- */

/* Housekeeping (the paper's workers read their partition of the training set, Section 5.1; here it is one
 * resident array).  Bind the training set resident in device memory: x_dev is [n_rows][dims[0]]
 * row-major, float for LS_GEMM_FP32 and bf16 for LS_GEMM_BF16 (16-byte aligned);
 * y_dev is int32[n_rows] class labels for LS_LOSS_SOFTMAX_CE (each in
 * [0, d_out)) or float[n_rows] targets for LS_LOSS_MSE_HALF.  Borrowed: must
 * stay valid while the handle uses it. */
int ls_bind_dataset(ls_handle* h, const void* x_dev, const void* y_dev, int64_t n_rows);

/* ---- the hot path ------------------------------------------------------ */

/* tau local updates on every replica, no communication (Section 2, PASGD
 * update rule, the case k mod tau != 0, applied tau times):
 *      for s = 0..tau-1, for every replica i independently:
 *          xi  = dataset rows [row_offset[s*m + i], + batch)
 *          g   = (1/|xi|) sum_{s in xi} grad f(x^(i); s)      (Section 2)
 *          v^(i) <- momentum * v^(i) + g ;  x^(i) <- x^(i) - lr * v^(i)
 * row_offset_host: host int64[tau][m], read before the call returns.
 * loss_dev: optional device float[tau][m]; entry [s][i] receives the mean loss
 * of replica i's mini-batch at step s, evaluated before that step's update.
 * Errors: tau < 1, NULL offsets, a batch outside the dataset. */
int ls_local_steps(ls_handle* h, int tau, const int64_t* row_offset_host, float* loss_dev);

/* One whole communication period: the tau local steps of ls_local_steps followed by
 * the averaging step of ls_average (Section 2, PASGD update rule: the update of
 * iteration k is averaged when k mod tau = 0), in one call.  The state after the
 * call is bit for bit the state after ls_local_steps(tau) then ls_average().
 * Arguments and errors as ls_local_steps. */
int ls_local_steps_avg(ls_handle* h, int tau, const int64_t* row_offset_host, float* loss_dev);

/* Same steps, but the mini-batches come from host memory and the losses go
 * back to host memory: x_host is [tau][m][batch][dims[0]] (float or bf16 as
 * for ls_bind_dataset), y_host [tau][m][batch] (int32 or float), loss_host
 * float[tau][m].  Pinned host memory lets the copies overlap the kernels of
 * the previous step.  Synchronous: returns when loss_host is filled. */
int ls_local_steps_host(ls_handle* h, int tau, const void* x_host, const void* y_host, float* loss_host);

/* Model averaging (Section 2, PASGD update rule, the case k mod tau = 0;
 * X <- X J with J = 1 1^T / m): every replica's parameters are replaced by the
 * mean over replicas; momentum buffers follow spec.momentum_mode.
 * The mean is defined to the bit: s = x^(0); s = s + x^(j) for j = 1..m-1 in
 * fp32, then one fp32 division by (float)m.  Afterwards all replicas are
 * bitwise equal.
 * LS_MOMENTUM_BLOCK: with `mean` as above, a the model the period started from
 * and u the global buffer (both kept in the state block, a = x_1 and u = 0 after
 * ls_set_params), in fp32 with every operation rounded on its own:
 *   d = a - mean;  G = d / lr;  u' = beta*u + G;  x' = a - lr*u'
 * x' replaces every replica's parameters and a, u' replaces u, the local
 * momentum buffers are cleared.  lr is the rate in force when ls_average runs. */
int ls_average(ls_handle* h);

/* ---- one job on several GPUs --------------------------------------------------
 * The paper's own layout (Section 2: m workers, models averaged "by a fusion node or by performing an
 * all-node broadcast"; its experiments ran one worker per GPU): the m_total replicas of a job are dealt out in
 * index order over n_gpus GPUs, one process and one handle per GPU, m = m_total / n_gpus replicas in each
 * handle.  Local steps need no communication.  The averaging step becomes
 *     p_g   = x^(0) + x^(1) + ... + x^(m-1)            on GPU g, over its own replicas in index order, fp32
 *     total = p_0 + p_1 + ... + p_{n_gpus-1}           in rank order, fp32, after ONE exchange that brings every
 *                                                      GPU's partial sum into this GPU's own memory
 *     mean  = total / (float)m_total                   written to every local replica
 * (the same for the momentum buffers in LS_MOMENTUM_AVERAGE).  This GROUPED order replaces the sequential
 * order of ls_average() on such a handle: it rounds differently for 1 < n_gpus < m_total, is identical for
 * n_gpus = 1, is fixed, and gives every GPU the same bits, so all m_total replicas end bitwise equal.
 * LS_MOMENTUM_BLOCK is not available on several GPUs (LS_ERR_UNSUPPORTED).
 *
 * The library links no communication library and never reads another GPU's memory: the exchange is the
 * caller's (an all-gather, e.g. NCCL through torch.distributed), handed over as a callback. */

/* exchange(ctx, partial_dev, gathered_dev, bytes, n_gpus): gathered_dev[g*bytes .. (g+1)*bytes) must receive
 * rank g's `bytes` bytes at partial_dev, for every g (this rank's own included).  The copy must be ordered
 * after the work already enqueued on the handle's stream and before anything enqueued on it afterwards
 * (enqueue the collective on that stream, or make the stream wait for it).  Returns 0 on success. */
typedef int (*ls_exchange_fn)(void* ctx, const float* partial_dev, float* gathered_dev, size_t bytes, int n_gpus);

/* Floats that partial_dev of ls_set_shard() must hold (two padded replica vectors: parameters and momentum);
 * gathered_dev holds n_gpus times as many. */
int ls_shard_buffer_floats(const ls_handle* h, int64_t* floats);

/* Declare that this handle's m replicas are rank-local shares of a job of m_total = n_gpus * m replicas.  From
 * then on every averaging step of the handle (ls_average, ls_local_steps_avg, the run loops) is the grouped
 * average above, with one call of `exchange` per averaging step.  partial_dev / gathered_dev: caller-allocated
 * device buffers (256-byte aligned, sizes above), borrowed until ls_destroy() or ls_set_shard(h, 0, ...).
 * n_gpus = 1 needs no callback (and equals ls_average() bit for bit); n_gpus = 0 switches back.
 * All ranks must call the hot-path functions in the same order (the exchange is collective); the controller
 * needs no exchange of its own: every rank evaluates the same synchronized model on the same probe rows and
 * reaches the same decision. */
int ls_set_shard(ls_handle* h, int n_gpus, int m_total, float* partial_dev, float* gathered_dev, ls_exchange_fn exchange,
                 void* ctx);

/* The two halves of the grouped average for callers that run the exchange themselves: the partial sums of this
 * handle's replicas into partial_dev, and, given all ranks' partial sums in rank order, the mean into every
 * local replica (momentum buffers as in ls_average). */
int ls_shard_partial_sum(ls_handle* h, float* partial_dev);
int ls_shard_average(ls_handle* h, const float* gathered_dev, int n_gpus, int m_total);

/* The same two kernels on raw buffers (32-byte aligned, strides multiples of 8 floats):
 * out_dev[0..P) = sum of the m vectors at buf_dev + j*stride in index order;
 * every one of the m_local vectors at dst_dev + j*dst_stride = (sum of the G vectors at
 * partials_dev + g*part_stride, in that order) / (float)m_total. */
int ls_partial_sum_flat(const float* buf_dev, int m, int64_t P, int64_t stride, float* out_dev, void* cuda_stream);
int ls_combine_partials_flat(const float* partials_dev, int G, int64_t part_stride, int m_total, int64_t P,
                             float* dst_dev, int m_local, int64_t dst_stride, void* cuda_stream);

/* Block-momentum state of a LS_MOMENTUM_BLOCK handle in the flat interface layout
 * (P floats each): the period-start model and the global buffer.  Either pointer
 * may be NULL.  Host memory; synchronous.  LS_ERR_UNSUPPORTED in other modes. */
int ls_set_block_state(ls_handle* h, const float* anchor_host, const float* u_host);
int ls_get_block_state(ls_handle* h, float* anchor_host, float* u_host);

/* The block-momentum averaging kernel on raw buffers: buf_dev as for
 * ls_average_flat, anchor_dev and u_dev vectors of P floats (device), lr > 0,
 * beta >= 0.  Same arithmetic as ls_average in LS_MOMENTUM_BLOCK. */
int ls_block_average_flat(float* buf_dev, float* anchor_dev, float* u_dev, int m, int64_t P, int64_t stride,
                          float lr, float beta, void* cuda_stream);

/* The averaging kernel on a raw buffer: m vectors of P floats, vector j
 * starting at buf_dev + j*stride floats (stride >= P).  Same arithmetic as
 * ls_average().  Fastest when buf_dev is 32-byte aligned and stride is a
 * multiple of 8 floats (256-bit accesses); 16-byte alignment and a stride
 * multiple of 4 give 128-bit accesses; anything else runs element by element. */
int ls_average_flat(float* buf_dev, int m, int64_t P, int64_t stride, void* cuda_stream);

/* Training loss of one replica on dataset rows [row_offset, +n_rows), the
 * empirical risk F of Section 2 restricted to those rows; n_rows must be a
 * positive multiple of `batch`.  Forward pass only.  Synchronous; writes one
 * host float. */
int ls_eval_loss(ls_handle* h, int replica, int64_t row_offset, int64_t n_rows, float* F_host);

/* AdaComm basic update rule (Section 4.2):
 *      tau_l = ceil( sqrt(F_t / F_0) * tau_0 ),   F_inf taken as 0,
 * evaluated in IEEE double exactly as written, clamped below at 1 (growth
 * above tau_0 is allowed).  Pure host function.  Returns the new period (>= 1)
 * or a negative LS_ERR_* (F_0 <= 0, F_t < 0, non-finite input, tau_0 < 1,
 * result beyond INT32_MAX). */
int adacomm_next_tau(double F_t, double F_0, int tau_0);

/* AdaComm with the refinements of Section 4.3:
 *   candidate (Section 4.3.2, learning-rate coupling)   c = ceil( sqrt( (lr_0/lr_l) * F_t/F_0 ) * tau_0 ), >= 1
 *   faster decay when training saturates (Section 4.3.1, slack s):
 *        tau_l = c  if c + slack < tau_prev,  else ceil(gamma * tau_prev), >= 1
 *   lr_changed != 0 (first decision after the learning rate changed): c is returned as it is, so the period
 *   may grow when the rate drops.
 * Pure host function, IEEE double.  Returns the period or a negative LS_ERR_* (non-finite input, F_0 <= 0,
 * F_t < 0, tau_0 < 1, tau_prev < 1, gamma outside (0, 1], slack < 0, a learning rate <= 0). */
int adacomm_next_tau_refined(double F_t, double F_0, int tau_0, int tau_prev, double gamma, int slack, double lr_0,
                             double lr_l, int lr_changed);

/* Options of ls_run_refined(). */
typedef struct ls_adacomm_opts {
  double gamma;              /* decay factor of Section 4.3.1, in (0, 1]; the paper uses 1/2 */
  int32_t slack;             /* slack variable s of Section 4.3.1, >= 0 */
  int32_t n_decay;           /* number of scheduled learning-rate decays */
  const int64_t* decay_at;   /* host, ascending: iteration counts at which a decay is scheduled */
  double decay_factor;       /* lr <- lr * decay_factor (the paper divides by 10) */
} ls_adacomm_opts;

/* ls_run() with the refined rules: the period is chosen by adacomm_next_tau_refined(), and a scheduled
 * learning-rate decay is applied at the first decision point at or past its iteration at which the period in
 * force is 1 (Section 4.3.2: let the period decay to 1 first); one decay per decision.  interval must be >= 1.
 * The handle's learning rate is changed by the decays (read it back with ls_get_lr()). */
int ls_run_refined(ls_handle* h, int64_t K, int tau_0, int interval, int64_t probe_rows,
                   const int64_t* row_offset_host, float* loss_dev, const ls_adacomm_opts* opts, int32_t* period_tau,
                   int64_t max_periods, int64_t* n_periods, int64_t* decision_k, float* decision_F,
                   int32_t* decision_tau, int64_t max_decisions, int64_t* n_decisions, float* F0_host);
int ls_get_lr(const ls_handle* h, float* lr);

/* Whole training run in native code: K local iterations cut into periods of
 * tau local steps, each followed by ls_average().  With interval > 0 the
 * period is re-chosen by adacomm_next_tau() at the first averaging point at or
 * past each multiple of `interval` iterations, from the loss of replica 0 on
 * dataset rows [0, probe_rows) (F_0 is that loss at the starting point);
 * interval == 0 keeps tau fixed.  A period is never cut by an interval
 * boundary; the last period is cut at K and averaged.
 * row_offset_host: int64[K][m].  loss_dev: optional device float[K][m].
 * Outputs (host, optional): period_tau[max_periods] / n_periods list the period
 * lengths requested; decision_k / decision_F / decision_tau [max_decisions] /
 * n_decisions log every AdaComm decision; F0_host the initial loss. */
int ls_run(ls_handle* h, int64_t K, int tau_0, int interval, int64_t probe_rows,
           const int64_t* row_offset_host, float* loss_dev,
           int32_t* period_tau, int64_t max_periods, int64_t* n_periods,
           int64_t* decision_k, float* decision_F, int32_t* decision_tau, int64_t max_decisions,
           int64_t* n_decisions, float* F0_host);

/* The same run with the intervals of Section 4 as the paper defines them: training is cut into
 * wall-clock intervals of length T0_ms, and the period is re-chosen at the first averaging point
 * after each interval boundary (the clock is the host's steady clock, read after the stream has
 * drained at every averaging point, starting when the first local step is enqueued).  The schedule
 * depends on how fast the machine is, so it is not reproducible; what is reproducible is that every
 * logged decision equals adacomm_next_tau(decision_F, F_0, tau_0).  T0_ms <= 0 decides at every
 * averaging point.  decision_ms (optional, [max_decisions]) receives the elapsed time of each decision. */
int ls_run_timed(ls_handle* h, int64_t K, int tau_0, double T0_ms, int64_t probe_rows,
                 const int64_t* row_offset_host, float* loss_dev,
                 int32_t* period_tau, int64_t max_periods, int64_t* n_periods,
                 int64_t* decision_k, float* decision_F, int32_t* decision_tau, double* decision_ms,
                 int64_t max_decisions, int64_t* n_decisions, float* F0_host);

/* ---- runtime model (host only; Sections 2-4) -------------------------------
 * The delay model and the runtime / error-runtime formulas that motivate the choice of the period.
 * Pure host functions: no GPU, no handle. */
enum { LS_DELAY_CONSTANT = 0, LS_DELAY_LOG2 = 1, LS_DELAY_TREE = 2, LS_DELAY_LINEAR = 3 };
/* D = D0 * s(m) with s(m) = 1, log2 m, 2 log2 m (reduction tree) or m  (Section 2, delay model). */
int ls_delay(double D0, int m, int scaling, double* D);
/* E[T_sync] / E[T_P-Avg] = (1 + alpha) / (1 + alpha / tau) for constant Y and D, alpha = D / Y (Section 3.2). */
int ls_speedup(double alpha, int tau, double* speedup);
/* Theorem 1: 2 (F1 - Finf) / (lr T) (Y + D / tau) + lr L sigma2 / m + lr^2 L^2 sigma2 (tau - 1). */
int ls_error_bound(double T, double F1, double Finf, double lr, double L, double sigma2, int m, int tau, double Y,
                   double D, double* bound);
/* Theorem 2: tau* = sqrt(2 (F1 - Finf) D / (lr^3 L^2 sigma2 T)). */
int ls_tau_star(double F1, double Finf, double D, double lr, double L, double sigma2, double T, double* tau);
/* Monte-Carlo means of the runtime per iteration (Section 3.1) over n_periods periods of tau local
 * steps of m workers: t_sync_mean of T_sync = max_i Y_i + D (every local step followed by a
 * broadcast), t_pavg_mean of T_P-Avg = max_i (sum_k Y_ik / tau) + D / tau, on the same draws.
 * Y_ik is exponential with mean y_mean (exponential != 0) or the constant y_mean.  The draw of
 * (period p, step k, worker i) is -y_mean ln((x + 0.5) / 2^32), x the first word of
 * Philox4x32-10(counter = (p lo, p hi, k, i), key = (seed lo, seed hi)). */
int ls_simulate_runtime(int m, int tau, int64_t n_periods, double y_mean, double D, uint64_t seed, int exponential,
                        double* t_sync_mean, double* t_pavg_mean);
/* One block of Philox4x32-10 (Salmon et al., SC'11). */
int ls_philox4x32_10(const uint32_t counter[4], const uint32_t key[2], uint32_t out[4]);

/* Mean loss of a linear model on device-resident rows, for callers that must not allocate.
 * (The paper has no counterpart: this entry point exists for deployment reasons only.)
 *
 * Some callers cannot obtain device memory when they need a loss value: code that runs inside a
 * memory pool owned by somebody else, a monitoring hook that fires when the device is nearly
 * full, a plugin that is forbidden to call cudaMalloc, code that must not disturb an allocator's
 * fragmentation state.  ls_eval_loss() needs the caller to have allocated a whole state block,
 * because the output-layer kernel keeps per-row losses, CTA counters and chunk offsets in
 * scratch memory.  Here that scratch is a fixed array inside the library image (about 260 KB of
 * every GPU that loads the library, held until the process exits), and the call allocates
 * nothing: no cudaMalloc, no cudaFree, no allocating library routine.
 *
 * Computes, for chunk c = 0 .. n_rows/chunk_rows - 1 of chunk_rows consecutive rows, the mean
 * loss of z = W x + b on those rows and writes it to chunk_loss_dev[c] (the caller's own device
 * buffer).  W_dev is float [d_out][d_in], bias_dev float [d_out] or NULL, x_dev float
 * [n_rows][d_in] (16-byte aligned for the fast path), y_dev int32 labels (LS_LOSS_SOFTMAX_CE) or
 * float targets (LS_LOSS_MSE_HALF, d_out == 1).  Same kernel and arithmetic as ls_eval_loss() on a
 * one-layer fp32 model with mini-batch chunk_rows.  Enqueued on cuda_stream; returns at once.
 *
 * Limits: d_out <= 16, at most 256 chunks and 65 536 rows per call, chunk_rows <= LS_MAX_BATCH;
 * beyond them the call returns LS_ERR_TOO_LARGE and does nothing.
 * The first call on each device looks up the scratch array's device address (with that device
 * current); make that first call outside any stream capture.
 * All calls on a device share the one scratch array: it keeps the previous call's contents (the
 * entry point re-clears what must start at zero), and two calls whose kernels overlap on the GPU
 * (different streams) race on it -- serialise them. */
int ls_linear_loss_static(const float* W_dev, const float* bias_dev, const float* x_dev, const void* y_dev,
                          int64_t n_rows, int d_in, int d_out, int loss, int chunk_rows, float* chunk_loss_dev,
                          void* cuda_stream);

/* ---- operators of a language model's blocks, last layers and weight update, on raw buffers ---------------------
 * Not passages of the paper: what a local-SGD job of a language model needs beside the averaging step.  Conventions:
 *  - m replicas in one call; *_stride is the distance in elements between replicas of that tensor (ignored for m == 1),
 *    inside a replica every tensor is dense and row-major.  Any size is allowed up to the limits stated; rows and
 *    replicas that start on 16-byte boundaries are read in vectors, others element by element.
 *  - dtype LS_DTYPE_*: the type of activations, operands and their gradients; sums, statistics and losses are fp32 or
 *    wider, and an output of dtype is rounded once.
 *  - ws_dev: the call's workspace, 256-byte aligned, at least *_ws_bytes() bytes (else LS_ERR_STATE_SIZE), contents
 *    irrelevant.  Two calls that may overlap on the GPU (other streams, other captured graphs) need workspaces of
 *    their own.  Nothing is kept in it between calls.
 *  - Enqueued on cuda_stream of the current device; the call returns at once and may be captured into a graph (the
 *    first call of an operator on a device outside any capture).  Results are the same bits on every run.
 *  - Outputs must not overlap inputs or each other.
 *  - Every wait inside a kernel is bounded; one that runs out is recorded per device and reported by
 *    ls_device_status().  The results of that call are invalid. */

/* Waits for cuda_stream, then returns LS_ERR_DEVICE_TIMEOUT once (and clears the record) if a wait of one of these operators ran
 * out on the current device since the last call, else LS_OK. */
int ls_device_status(void* cuda_stream);
/* Housekeeping: ls_selftest_wait_timeout() for this report path.  The kernel records its failure like an operator on the
 * current device would: the next ls_device_status() returns LS_ERR_DEVICE_TIMEOUT, the one after it LS_OK. */
int ls_selftest_device_timeout(int64_t limit_cycles, void* cuda_stream);

/* Layer norm of every row of x [m][rows][d]:  y = (x - mean) * rstd * weight + bias,  rstd = 1 / sqrt(var + eps), var the
 * mean square of x - mean.  weight, bias (may be NULL): float [m][d], param_stride apart.  y like x.  mean, rstd
 * (either may be NULL): float [m][rows], dense.  eps >= 0.  d <= 16384. */
int ls_layer_norm(const void* x_dev, const float* weight_dev, const float* bias_dev, int m, int64_t rows, int d,
                  int64_t x_stride, int64_t param_stride, int dtype, float eps, void* y_dev, int64_t y_stride,
                  float* mean_dev, float* rstd_dev, void* cuda_stream);

/* Its gradient, from dy, x and the mean and rstd that the forward call wrote:
 *   dx = rstd * (t - <t> - xhat <t xhat>),  t = dy * weight, xhat = (x - mean) * rstd, <.> the mean over a row,
 *   dweight = sum over rows of dy * xhat,  dbias (may be NULL) = sum over rows of dy
 * dweight, dbias: float [m][d], dparam_stride apart, overwritten (zeros for rows == 0). */
int ls_layer_norm_grad_ws_bytes(int m, int64_t rows, int d, size_t* bytes);
int ls_layer_norm_grad(const void* dy_dev, const void* x_dev, const float* weight_dev, const float* mean_dev,
                       const float* rstd_dev, int m, int64_t rows, int d, int64_t dy_stride, int64_t x_stride,
                       int64_t param_stride, int dtype, void* dx_dev, int64_t dx_stride, float* dweight_dev,
                       float* dbias_dev, int64_t dparam_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream);

/* Softmax cross entropy of the logits h W^T of a wide output matrix, without storing the logits:
 *   z_n = W h_n,  lse_n = log sum_v exp z_nv,  row_loss_n = lse_n - z_n,y(n),  loss = mean of row_loss over labelled rows
 * h [m][rows][d], W [m][vocab][d] of dtype; labels int32 [m][rows], dense: a label outside [0, vocab) marks a row
 * without one (padding), whose row_loss is 0 and which does not count (loss is 0 when no row counts).
 * loss float [m]; row_loss, lse float [m][rows], dense, either may be NULL.
 * vocab <= 2^24, d <= 65536.  When a row is whole 16-byte pieces (d a multiple of 8 for bf16, 4 for fp32), h, W, dh, dW
 * and their strides must be 16-byte multiples (else LS_ERR_INVALID_ARG).
 * In fp32 an infinite element of h or W counts as 3.39e38 with its sign.
 * Workspace of the loss: two numbers a row and slice of 64 or 128 columns (and a copy of both operands for fp32 or d not
 * a multiple of 8).  Of the gradient: also the probabilities of a piece of rows, at most about 1 GiB but at least 256
 * rows, h of that piece, and the fp32 sum of dW for bf16 when the rows take several pieces.  Where all of that stays below
 * 512 MB for all replicas, they are taken together.  A workspace of the gradient's size serves the loss of the same sizes, too. */
int ls_vocab_loss_ws_bytes(int m, int64_t rows, int64_t vocab, int d, int dtype, int grad, size_t* bytes);
int ls_vocab_loss(const void* h_dev, const void* W_dev, const int32_t* labels_dev, int m, int64_t rows, int64_t vocab,
                  int d, int64_t h_stride, int64_t w_stride, int dtype, float* loss_dev, float* row_loss_dev,
                  float* lse_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream);

/* The same losses, and the gradients of scale * loss: dh [m][rows][d] (zero in rows without a label, if W is finite),
 * dW [m][vocab][d], both of dtype, overwritten.  h of rows without a label does not enter dW, whatever it holds.
 * bf16: the gradient of the logits, an operand of both products, is rounded to bf16 (2^-8 of each of its numbers, down to 43 nats
 * below the largest of its 64 or 128 neighbours), except for up to 4 rows with d a multiple of 8. */
int ls_vocab_loss_grad(const void* h_dev, const void* W_dev, const int32_t* labels_dev, int m, int64_t rows, int64_t vocab,
                       int d, int64_t h_stride, int64_t w_stride, int dtype, float scale, float* loss_dev,
                       float* row_loss_dev, float* lse_dev, void* dh_dev, int64_t dh_stride, void* dW_dev,
                       int64_t dw_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream);

/* Orthogonalisation of the matrices u [m][rows][cols] by `steps` (1..64) Newton-Schulz steps:
 *   X = u / (|u|_F + 1e-7);  repeat: A = X X^T, X = 3.4445 X + (-4.7750 A + 2.0315 A A) X;  out = X
 * (for rows > cols the same of the transpose, transposed back).  Products are accurate to about 22 bits, and from fp32 numbers
 * the result is as far from the formula's as fp32 arithmetic leaves it (1e-6 to 4e-6 of the norm).  From bf16 numbers
 * two or three steps of a large matrix longer than wide may be taken together (A of the first, A' = A P P after that),
 * which is off by some 1e-6 of the result's norm, 2e-5 where singular values span decades.  |u|_F is added up in double; a matrix whose
 * norm is not large against 1e-7 comes out smaller, as the formula has it.  out has u's dtype and shape.
 * rows, cols <= 32768.  The workspace also serves ls_muon_step. */
int ls_orthogonalize_ws_bytes(int m, int rows, int cols, size_t* bytes);
int ls_orthogonalize(const void* u_dev, int m, int rows, int cols, int64_t u_stride, int dtype, int steps, void* out_dev,
                     int64_t out_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream);

/* One orthogonalised momentum step (the Muon update) of the matrices w [m][rows][cols] with momentum buffers v, both
 * fp32, in the caller's memory (for the weights of a handle: ls_muon_step_layer()), from gradients g of g_dtype:
 *   v <- momentum * v + g;   u = nesterov ? g + momentum * v : v;   w <- w - lr * sqrt(max(1, rows / cols)) * O(u)
 * with O the orthogonalisation above.  0 <= momentum < 1. */
int ls_muon_step(float* w_dev, float* v_dev, const void* g_dev, int m, int rows, int cols, int64_t w_stride,
                 int64_t v_stride, int64_t g_stride, int g_dtype, float lr, float momentum, int nesterov, int steps, void* ws_dev,
                 size_t ws_bytes, void* cuda_stream);

/* The same step of the matrix W_l of layer `layer` (0-based) of all m replicas of a handle, with the handle's momentum
 * buffers as v, from gradients g [m][dims[layer + 1]][dims[layer]], row-major, g_stride elements apart.  Whatever the
 * handle keeps beside the weights follows: local steps, averages and losses after the call see the new weights.  Biases stay as
 * they are; lr and momentum are this call's own, not the handle's.  Enqueued on the handle's stream, and not to
 * be captured into a graph (LS_ERR_UNSUPPORTED); workspace as ls_orthogonalize_ws_bytes(m, dims[layer + 1], dims[layer]) has it.
 * A wait that runs out is reported by ls_device_status(), not by ls_sync(). */
int ls_muon_step_layer(ls_handle* h, int layer, const void* g_dev, int64_t g_stride, int g_dtype, float lr, float momentum,
                       int nesterov, int steps, void* ws_dev, size_t ws_bytes);

/* RMS norm of every head of q and k and rotation by position, in one pass:
 *   z = x / sqrt(mean of x^2 over the head + eps) * weight,  then the pairs of the first rot_dim elements of z are turned:
 *   (a, b) -> (a cos - b sin, a sin + b cos),  angle = positions[token] * inv_freq[pair]
 * Pair p is the elements (p, p + rot_dim / 2), or (2 p, 2 p + 1) when interleaved; the other elements stay as they are.
 * q [m][tokens][heads][head_dim], k [m][tokens][kv_heads][head_dim], and their outputs, of dtype: *_row is the distance in
 * elements between tokens of a tensor, *_stride that between replicas, one behind the other (ignored for one token, one replica), the heads of a
 * token are dense, so that q and k may be parts of one projection.  weights: float [m][head_dim], weight_stride apart.
 * inv_freq: double [rot_dim / 2], positions: int32 [m][tokens], dense (either may be NULL if rot_dim == 0).  Angles
 * are formed in double, squares and their mean in fp32 (elements of up to 10^18).  rot_dim is even.  head_dim <= 256, tokens <=
 * 2^30, heads <= 65536. */
int ls_qk_norm_rope(const void* q_dev, const void* k_dev, const float* q_weight_dev, const float* k_weight_dev,
                    const int32_t* positions_dev, const double* inv_freq_dev, int m, int64_t tokens, int heads, int kv_heads,
                    int head_dim, int rot_dim, int interleaved, int64_t q_row, int64_t k_row, int64_t q_stride, int64_t k_stride,
                    int64_t weight_stride, int dtype, float eps, void* q_out_dev, void* k_out_dev, int64_t q_out_row,
                    int64_t k_out_row, int64_t q_out_stride, int64_t k_out_stride, void* cuda_stream);

/* Its gradient, from the gradients of both outputs and the call's inputs: dq, dk like q and k (in rows of their own distances), and
 * dq_weight, dk_weight: float [m][head_dim], dweight_stride apart, sums over tokens and heads, overwritten (zeros for no tokens). */
int ls_qk_norm_rope_grad_ws_bytes(int m, int64_t tokens, int head_dim, size_t* bytes);
int ls_qk_norm_rope_grad(const void* dq_out_dev, const void* dk_out_dev, const void* q_dev, const void* k_dev,
                         const float* q_weight_dev, const float* k_weight_dev, const int32_t* positions_dev,
                         const double* inv_freq_dev, int m, int64_t tokens, int heads, int kv_heads, int head_dim, int rot_dim,
                         int interleaved, int64_t dq_out_row, int64_t dk_out_row, int64_t q_row, int64_t k_row,
                         int64_t dq_out_stride, int64_t dk_out_stride, int64_t q_stride, int64_t k_stride, int64_t weight_stride,
                         int dtype, float eps, void* dq_dev, void* dk_dev, int64_t dq_row, int64_t dk_row, int64_t dq_stride,
                         int64_t dk_stride, float* dq_weight_dev, float* dk_weight_dev, int64_t dweight_stride, void* ws_dev,
                         size_t ws_bytes, void* cuda_stream);

/* Causal attention over packed sequences, without stored scores:
 *   s_ij = scale q_i . k_j  over the keys j <= i of i's own sequence,  out_i = sum_j softmax(s_i)_j v_j,  lse_i = log sum_j exp s_ij
 * q, out [m][tokens][heads][head_dim], k, v [m][tokens][kv_heads][head_dim] of dtype, rows and replicas apart as for
 * ls_qk_norm_rope; heads is a multiple of kv_heads, and head h reads key head h / (heads / kv_heads).
 * seq_start: int32 [m][n_seqs + 1], dense, ascending: sequence s of a replica is the rows [seq_start[s], seq_start[s + 1]), of any
 * length, none included.  NULL with n_seqs == 1: one sequence of all rows.  Rows in no sequence (before the first, behind the
 * last) get out = 0 and lse = 0, and whatever they hold reaches no other row; nor does a NaN reach another sequence or an
 * earlier row of its own.  (Boundaries that do not ascend or leave [0, tokens] give wrong results, but no access outside, and no wait runs out.)
 * lse: float [m][heads][tokens], dense.  A row whose scores are all -inf, or one +inf, has no softmax: its out is NaN.
 * bf16 on the tensor cores (head_dim a multiple of 8 up to 128, every row of every tensor on a 16-byte boundary, scale > 0):
 * probabilities are rounded to bf16 as the operand of the second product, their sum is not.  Other calls run on the CUDA cores.
 * head_dim <= 256, tokens <= 2^30. */
int ls_attention(const void* q_dev, const void* k_dev, const void* v_dev, const int32_t* seq_start_dev, int m, int64_t tokens,
                 int n_seqs, int heads, int kv_heads, int head_dim, int64_t q_row, int64_t k_row, int64_t v_row, int64_t q_stride,
                 int64_t k_stride, int64_t v_stride, int dtype, float scale, void* out_dev, int64_t out_row, int64_t out_stride,
                 float* lse_dev, void* cuda_stream);

/* Its gradient, from dout, the inputs, and the out and lse that the forward call wrote:
 *   P_ij = exp(s_ij - lse_i),  dS_ij = P_ij (dout_i . v_j - dout_i . out_i),
 *   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dout_i
 * dk and dv sum over the query heads of their group.  Zero for rows in no sequence, whose dout may hold anything.  Where the
 * tensor cores take the call (see above), P and dS are rounded to bf16 as operands of dv and dk; of dq, dS is two bf16 pieces. */
int ls_attention_grad_ws_bytes(int m, int64_t tokens, int heads, int kv_heads, int head_dim, size_t* bytes);
int ls_attention_grad(const void* dout_dev, const void* q_dev, const void* k_dev, const void* v_dev, const void* out_dev,
                      const float* lse_dev, const int32_t* seq_start_dev, int m, int64_t tokens, int n_seqs, int heads, int kv_heads,
                      int head_dim, int64_t dout_row, int64_t q_row, int64_t k_row, int64_t v_row, int64_t out_row,
                      int64_t dout_stride, int64_t q_stride, int64_t k_stride, int64_t v_stride, int64_t out_stride, int dtype,
                      float scale, void* dq_dev, void* dk_dev, void* dv_dev, int64_t dq_row, int64_t dk_row, int64_t dv_row,
                      int64_t dq_stride, int64_t dk_stride, int64_t dv_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream);

/* The global norm of every replica's gradients, and clipping to it:
 *   norm[r] = sqrt(sum over all tensors of replica r of g^2),  g <- g if norm[r] <= max_norm, else g * (max_norm / norm[r])
 * Host arrays of n_tensors entries: tensor i has sizes[i] elements a replica, of dtypes[i], strides[i] apart (dense within a
 * replica; strides may be NULL for m == 1).  outs NULL: in place; else the results go to outs[i] (of out_dtypes[i], rounded once,
 * out_strides[i] apart; grads[i] itself, with its type and stride, is allowed) and gradients that are not their own outputs stay.
 * An output that shares memory with another output, or with a gradient that is not its own, is refused (LS_ERR_INVALID_ARG).
 * norm: float [m].  max_norm > 0; INFINITY: the norm, and nothing is scaled.  A norm of NaN makes the replica's results NaN;
 * that of an infinite gradient makes them 0, and NaN where a gradient is infinite.  Sums are formed in double over fp32 sums of 32 squares; no
 * square overflows or underflows, and a finite norm beyond fp32's largest number is written as infinity, but clips as what it is.  The arrays are read before the call returns.  n_tensors <= 65536. */
int ls_clip_grads_ws_bytes(const int64_t* sizes, int n_tensors, int m, size_t* bytes);
int ls_clip_grads(const void* const* grads_dev, const int64_t* sizes, const int64_t* strides, const int32_t* dtypes, int n_tensors,
                  int m, double max_norm, void* const* outs_dev, const int64_t* out_strides, const int32_t* out_dtypes,
                  float* norm_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream);

/* Per-kernel device timing.  Between ls_profile_begin() and ls_profile_end()
 * every launch of a kernel class selected by class_mask (bit c = class c; for
 * the per-layer classes only layer `layer`, 0-based, or all layers when
 * layer < 0) is bracketed by a pair of CUDA events on the handle's stream.
 * ls_profile_end() waits for the stream and adds up, per class and layer, the
 * elapsed milliseconds and the number of launches into
 * ms[LS_K_CLASSES * LS_MAX_LAYERS] and launches[...] (index class*LS_MAX_LAYERS
 * + layer; LS_K_LOSS uses layer 0; LS_K_AVG uses layer 0 for the averaging
 * kernel and layer 1 for the launch that does the last weight update of a
 * period and its averaging step together, both whatever `layer` says).  At most
 * 16384 launches are recorded per profile; later ones are run but not timed. */
enum { LS_K_FWD = 0, LS_K_LOSS = 1, LS_K_DX = 2, LS_K_DW = 3, LS_K_BIAS = 4, LS_K_AVG = 5, LS_K_CLASSES = 6 };
int ls_profile_begin(ls_handle* h, uint32_t class_mask, int layer);
int ls_profile_end(ls_handle* h, double* ms, int64_t* launches);

/* Number of kernels this handle has launched so far. */
int ls_launch_count(const ls_handle* h, int64_t* n);

#ifdef __cplusplus
}
#endif
#endif /* LS_H_ */
