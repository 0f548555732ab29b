/*
 * combo_b200 -- one synchronization round of segmented gossip aggregation
 * ("Decentralized Federated Learning: A Segmented Gossip Approach") for N
 * simulated workers whose flat parameter vectors sit in one GPU's memory.
 *
 * C ABI of libcombo_b200.so (CUDA, sm_100a only; there is no CPU or other
 * fallback).  Plain pointers and sizes; the caller owns every buffer.  Unless
 * a function says otherwise, pointers are DEVICE pointers of the current
 * device, calls only enqueue work on the given stream and never synchronise,
 * and the library allocates nothing.
 *
 * Library-owned device memory: a 4-byte status word (combo_device_status) and
 * a ring of 256 tile dispensers, 16 bytes each.  Every launch of the staged
 * aggregation kernel with persistent CTAs takes the next dispenser (its CTAs
 * draw their tiles from it and the last one to leave clears it): ordinary
 * launches cycle through one half of the ring, launches that are being
 * captured into a CUDA graph through the other half.  Ordinary launches in
 * flight at the same time therefore hold different dispensers as long as
 * fewer than 128 staged launches separate them, and a graph replay never
 * shares one with ordinary launches running beside it.  A graph keeps the
 * dispensers it was captured with: two replays (of one graph or of different
 * ones) whose staged kernels could run at the same time must not hold the
 * same dispenser -- do not run a graph concurrently with itself, nor with a
 * graph captured a multiple of 128 staged launches before or after it.
 * Sharing a dispenser loses or repeats tiles (wrong output, no fault).
 *
 * Notation follows the paper: n = N workers, S segments, R model replicas,
 * |D_j| dataset size of worker j, P_l the set of workers providing segment l.
 *
 * Layouts
 *   parameters  [N][P] row-major, worker-major, dense (row pitch = P elements)
 *   idx         int32 [N][S][R]; idx[w][l][r] = r-th peer of worker w for
 *               segment l; each (w,l) row ascending, all entries != w, distinct
 *   weights     float [N], |D_j| > 0, un-normalised; NULL = all equal
 *
 * Segments (Eq. 1; Section 5.1 cuts the model into S equal parts): segment
 * length L = ceil(P/S); segment l covers columns [min(l*L,P), min((l+1)*L,P)),
 * so the last segment is shorter when S does not divide P and trailing
 * segments may be empty.
 */
#ifndef COMBO_B200_H
#define COMBO_B200_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int combo_status;

enum {
    COMBO_OK = 0,                 /* work enqueued (or, for host calls, done)    */
    COMBO_ERR_INVALID_ARG = 1,    /* size out of range, NULL or misaligned pointer */
    COMBO_ERR_ALIAS = 2,          /* input and output ranges overlap             */
    COMBO_ERR_UNSUPPORTED = 3,    /* current device is not compute capability 10.x */
    COMBO_ERR_CUDA = 4,           /* a CUDA runtime call failed; see combo_last_cuda_error */
    COMBO_ERR_DEVICE_TIMEOUT = 5, /* a bounded wait inside a kernel ran out      */
    COMBO_ERR_TOO_LARGE = 6       /* beyond the fixed limit of a no-allocation entry point */
};

/* Limits of this library version. */
#define COMBO_MAX_WORKERS 8192    /* N */
#define COMBO_MAX_SEGMENTS 65536  /* S */
#define COMBO_NOALLOC_MAX_WORKERS 128   /* N of combo_aggregation_divergence_noalloc */

/*
 * Peer selection -- Section 4.1, step (2) "Segments Pulling": every worker
 * issues S*R pull requests; each target is drawn at random from all the OTHER
 * workers, without replacement, until no option is left.  When the pool of
 * N-1 others is exhausted a freshly shuffled pool is opened; peers already
 * chosen for the segment being filled are skipped (P_l of Eq. 3 is a set).
 * Hence: never the worker itself, R distinct peers per (worker, segment), all
 * S*R peers of a worker distinct when S*R <= N-1, otherwise every other worker
 * is used floor or ceil of S*R/(N-1) times.
 *
 * The table is a pure function of (seed, round, N, S, R): random numbers come
 * from a counter-based generator (splitmix64 steps chained over the words
 * seed, round|worker, epoch|position; Fisher-Yates shuffle with the
 * multiply-shift range reduction), so the call can be issued ahead of the
 * local update, as the paper notes for the pull requests.
 *
 * idx_out: device int32[N*S*R], written completely; not touched when R == 0.
 * Requires 1 <= N <= COMBO_MAX_WORKERS, 1 <= S <= COMBO_MAX_SEGMENTS,
 * 0 <= R <= N-1.  combo_select_peers enqueues on the legacy default stream;
 * the _async form on `stream` (a cudaStream_t passed as void*).
 */
combo_status combo_select_peers(uint64_t seed, uint32_t round, int N, int S, int R,
                                int32_t* idx_out);
combo_status combo_select_peers_async(uint64_t seed, uint32_t round, int N, int S, int R,
                                      int32_t* idx_out, void* stream);

/*
 * Segment-wise aggregation -- Eq. 3 and Eq. 4 (Section 3, "Segmented
 * Aggregation"), for all N workers at once:
 *
 *   out[w][p] = sum_{j in P_l(w)} |D_j| * in[j][p]  /  sum_{j in P_l(w)} |D_j|
 *
 * with l the segment that holds column p and P_l(w) = {w} U idx[w][l][0..R).
 * Every worker reads the same pre-aggregation inputs (workers send the model
 * they hold after the local update, Section 4.1 steps 3 and 4), so params_out
 * must not overlap params_in.
 *
 * Arithmetic: binary32, Eq. 3 as it is written.  num = |D_w|*x_w, then
 * num = fma(|D_k|, x_k, num) for the peers in ascending order;
 * den = |D_w| + |D_k1| + ... in the same order; out = num * (1/den), the
 * reciprocal rounded to binary32 (one IEEE division per worker and segment).
 * A single provider is taken as it is (out = x).  With weights == NULL every
 * |D_j| is 1: the products are exact and num is the plain sum in that order
 * (bfloat16 rows are then added by the mixed-precision instruction
 * add.rn.f32.bf16, which widens exactly and rounds once: the same bits).
 * |D_j|*x must stay within the binary32 range.  No fast-math, denormals kept.
 *
 * params_in, params_out: float [N][P], base addresses 16-byte aligned.
 * weights: float[N] or NULL.  idx: int32[N][S][R], trusted (see
 * combo_validate_idx); may be NULL when R == 0.  1 <= P, 0 <= R <= N-1.
 * R == 0 copies the input bit for bit.
 */
combo_status combo_segment_aggregate(const float* params_in, float* params_out,
                                     const float* weights, const int32_t* idx,
                                     int N, int64_t P, int S, int R, void* stream);

/*
 * The same with parameters stored as bfloat16 (uint16_t bit patterns):
 * inputs are widened exactly, accumulation is binary32 as above, the result
 * is rounded to nearest even.  Rows need not be 16-byte aligned (odd P*2
 * pitches are handled); the base addresses must be.
 */
combo_status combo_segment_aggregate_bf16(const uint16_t* params_in, uint16_t* params_out,
                                          const float* weights, const int32_t* idx,
                                          int N, int64_t P, int S, int R, void* stream);

/*
 * Local step fused in front of the aggregation -- Section 4.1 step (1) with
 * one SGD step (tau = 1) on a supplied gradient: every worker j first forms
 * x'_j = fma(-lr, grads[j], params_in[j]) (binary32), and Eq. 3 is evaluated
 * on the x'.  Peers contribute their UPDATED rows, exactly as if the step had
 * been applied to all of params_in before combo_segment_aggregate.  grads:
 * float [N][P], 16-byte aligned, must not overlap params_out.
 */
combo_status combo_segment_aggregate_sgd(const float* params_in, const float* grads, float lr,
                                         float* params_out, const float* weights,
                                         const int32_t* idx, int N, int64_t P, int S, int R,
                                         void* stream);

/*
 * Column-sharded form of the three calls above, for a vector of P_total
 * parameters whose columns [p_begin, p_begin + width) are held locally as
 * [N][pitch] arrays (pitch >= width elements; local column 0 = global column
 * p_begin).  Eq. 3 couples workers only at equal p, so shards need no
 * exchange; segment bounds are those of the P_total-vector.
 * elem_bytes: 4 = float, 2 = bfloat16.  grads may be NULL (no local step;
 * must be NULL for bfloat16).
 */
combo_status combo_segment_aggregate_cols(const void* params_in, const void* grads, float lr,
                                          void* params_out, int elem_bytes,
                                          const float* weights, const int32_t* idx,
                                          int N, int64_t P_total, int S, int R,
                                          int64_t p_begin, int64_t width, int64_t pitch,
                                          void* stream);

/*
 * Worker-sharded form -- Section 3 "Segmented Pulling" (Eq. 2) followed by
 * Eq. 3, for workers spread over several GPUs of one node.  d_rows: DEVICE
 * array of N pointers, d_rows[j] = flat model of worker j (P elements, 16-byte
 * aligned), in this GPU's memory or in a peer GPU's memory that is mapped
 * into this process (peer access / symmetric memory).  The call forms the new
 * models of the n_local workers w_begin .. w_begin + n_local - 1 that this
 * GPU hosts and writes them to out, [n_local][out_pitch] (out_pitch >= P
 * elements, out_pitch * elem_bytes a multiple of 16; must not overlap any
 * row).  A pull is a plain load of W_k[l] from where worker k lives (no bulk
 * copy, no multicast); a segment of a peer that several hosted workers pull
 * is loaded once per column tile and shared, so per segment index at most R
 * segments per hosted worker cross to this GPU -- the paper's count, less the
 * shared ones.  idx is the full [N][S][R] table (every GPU computes the same
 * one from the seed), weights the full [N] array or NULL.  Same arithmetic and
 * order as combo_segment_aggregate.  The caller orders the rounds: rows must
 * be final before the call (Section 4.1: a worker sends after its local
 * update) and must not be overwritten while any GPU still reads them.
 */
combo_status combo_segment_aggregate_rows(const void* const* d_rows, void* out, int64_t out_pitch,
                                          int elem_bytes, const float* weights, const int32_t* idx,
                                          int N, int64_t P, int S, int R, int w_begin, int n_local,
                                          void* stream);

/* Debug helper for the call above: *dev_flag (device int32) becomes 0 when all
 * N row pointers are non-null and 16-byte aligned, else 1 + the first bad row. */
combo_status combo_check_rows(const void* const* d_rows, int N, void* stream, int32_t* dev_flag);

/*
 * Dynamic workers -- Section 4.2.
 *
 * combo_select_peers_online: a worker that is offline is not pulled from (its
 * requester turns to some other worker instead), so every online worker
 * draws its peers from the ONLINE others only, by the same procedure as
 * combo_select_peers (identical tables when all are online).  An offline worker
 * issues no requests: its rows are filled with -1.  h_online: HOST array of N
 * bytes, non-zero = online (membership is decided on the host); NULL = all
 * online.  Requires R <= (online workers) - 1.
 *
 * combo_segment_aggregate_members: Eq. 3 with the provider set
 *   P_l(w) = ({w} unless w is a newcomer) U { idx[w][l][r] : idx[w][l][r] >= 0 }.
 * A newcomer has no model of its own yet: it aggregates the segments it
 * pulled without an own term (Section 4.2), so its row is never read; a
 * negative idx entry is a pull that found no online peer.  A worker left with no provider (an offline
 * worker's -1 rows) keeps its own values.  h_newcomer: HOST array of N bytes,
 * non-zero = newcomer, or NULL.  Same arithmetic and order as
 * combo_segment_aggregate (providers in the order self, peers ascending); all
 * entry points above accept negative idx entries in the same way (the
 * worker-sharded call too; it has no newcomer flags).  Rows that are read must
 * hold finite values.
 */
combo_status combo_select_peers_online(uint64_t seed, uint32_t round, int N, int S, int R,
                                       const uint8_t* h_online, int32_t* idx_out, void* stream);
combo_status combo_segment_aggregate_members(const void* params_in, void* params_out, int elem_bytes,
                                             const float* weights, const int32_t* idx,
                                             const uint8_t* h_newcomer, int N, int64_t P, int S, int R,
                                             void* stream);

/*
 * Checks an idx table on the device: every entry in [0,N), != its worker,
 * each (w,l) row strictly ascending.  dev_flag: device int32, set to 0 first,
 * then to 1 + (index of an offending entry) if any check fails.
 */
combo_status combo_validate_idx(const int32_t* idx, int N, int S, int R, void* stream,
                                int32_t* dev_flag);

/*
 * Whole rounds from HOST memory (the paper's worker iteration, steps 2-4, for
 * all workers): copies h_params_in (and h_grads, h_weights when given) to the
 * device buffers, then for t = round .. round+rounds-1 selects peers for
 * (seed, t) and aggregates, ping-ponging between d_in and d_out, and copies
 * the final parameters to h_params_out; all on `stream`, which is
 * synchronised before returning.  With h_grads the fused local step uses the
 * same gradient array in every round.  Host buffers should be page-locked
 * for full copy speed.  Device buffers are the caller's: d_in, d_out (and
 * d_grads if h_grads != NULL) [N][P] of elem_bytes each, d_weights float[N]
 * (if h_weights != NULL), d_idx int32[N*S*R].  h_idx_out, if not NULL,
 * receives the peer table of the last round.  rounds >= 1.
 * Columns are independent in Eq. 3, so the call cuts the vector into column
 * chunks and overlaps the copy-in of one chunk, all rounds of the previous
 * one and the copy-out of the one before on three streams (two of them, and
 * a few events, are created by the first call on a device and kept).  Not
 * reentrant per device.  After the call d_in and d_out hold intermediate
 * rounds, not a defined result.
 */
combo_status combo_round_host(const void* h_params_in, const void* h_grads, float lr,
                              void* h_params_out, int elem_bytes, const float* h_weights,
                              uint64_t seed, uint32_t round, int rounds, int N, int64_t P, int S,
                              int R, void* d_in, void* d_grads, void* d_out, float* d_weights,
                              int32_t* d_idx, int32_t* h_idx_out, void* stream);

/*
 * Aggregation divergence -- Section 4.3, Definition 2 (Eq. 7): for every
 * worker i, rho_i = || W_{t,i} - W_t || (Euclidean norm), where W_{t,i} is row
 * i of `models` (the worker's aggregation result) and W_t is the aggregation
 * of ALL workers, the FedAvg result sum_j |D_j| W_j / sum_j |D_j|, taken over
 * the rows of `mean_of` (the models the round started from).  mean_of == NULL
 * or == models measures the models against their own weighted mean.  With
 * R = N-1 every rho_i is zero up to rounding, as the paper states.
 *
 * models, mean_of: [N][P] dense, elem_bytes 4 (float) or 2 (bfloat16), read
 * only.  rho_out: device double[N].  scratch: device memory of at least
 * combo_divergence_scratch_bytes(N) bytes, 8-byte aligned, used for per-CTA
 * partial sums (no need to clear it; contents are undefined afterwards).
 * Arithmetic: column means and deviations in binary32 (weights normalised
 * first, rows in ascending order), squares summed in binary64; relative error
 * of rho about 1e-6 for models that differ by more than 1e-3 of their size.
 * Two launches on `stream`, no synchronisation.
 */
size_t combo_divergence_scratch_bytes(int N);
combo_status combo_aggregation_divergence(const void* models, const void* mean_of, int elem_bytes,
                                          const float* weights, int N, int64_t P, double* rho_out,
                                          void* scratch, size_t scratch_bytes, void* stream);

/*
 * combo_aggregation_divergence for callers that cannot allocate device memory.
 * (The paper has no counterpart: this is a packaging variant of the call above,
 * same arithmetic, same result.)
 *
 * Who needs it: code that runs where cudaMalloc is not an option -- inside a
 * region being captured into a CUDA graph or between other work that must not
 * synchronise the device (cudaMalloc and cudaFree may do both), in a process
 * whose memory pool is owned and fully handed out by another component, or
 * in a host language binding that cannot create device buffers at all.  Such
 * a caller still passes its inputs and the output, but no scratch: the
 * partial sums go to a fixed array inside the library, 1 MiB that every GPU
 * loading the library holds until the process exits.
 *
 * Limits and rules:
 *  - N <= COMBO_NOALLOC_MAX_WORKERS (128); more returns COMBO_ERR_TOO_LARGE
 *    and combo_last_cuda_error() says so.  P is not limited.
 *  - The first call on each device looks the array's device address up
 *    (cudaGetSymbolAddress, with that device current) and keeps it; make that
 *    first call outside any stream capture.  No call allocates or frees.
 *  - All calls on a device share the one array and it keeps whatever the last
 *    call left.  Nothing has to be cleared, because every partial sum is
 *    written before it is read; but two calls that overlap on the GPU (other
 *    streams, other host threads) race on it -- serialise them on one stream.
 */
combo_status combo_aggregation_divergence_noalloc(const void* models, const void* mean_of,
                                                  int elem_bytes, const float* weights, int N,
                                                  int64_t P, double* rho_out, void* stream);

/*
 * ---------------------------------------------------------------------------
 * The local step (Section 4.1 step (1)) for all workers at once: the operators
 * that lead from a worker's samples to the gradient combo_segment_aggregate_sgd
 * takes.  The paper trains with a framework's layers and states none of these;
 * their formulas stand here.
 * ---------------------------------------------------------------------------
 *
 * Gradient norms over many tensors, and clipping.  Worker w's gradient is a list
 * of tensors; norm_w is taken over all of them together, and
 *
 *   norm_w = sqrt( sum g^2 ),   c_w = min(1, max_norm / (norm_w + 1e-6)),   out = c_w * g
 *
 * d_tensors: DEVICE array of n_tensors addresses, each aligned to its element
 * (elem_bytes 4 = float, 2 = bfloat16), in the workers' order.  d_begin: device
 * int64[n_tensors + 1], d_begin[t] = number of elements in the tensors before t
 * (d_begin[0] = 0, d_begin[n_tensors] = total).  d_first: device int32[N + 1],
 * worker w owns tensors d_first[w] .. d_first[w+1] - 1 (d_first[0] = 0,
 * d_first[N] = n_tensors).  Tensors and workers may be empty.  The three arrays
 * are trusted, like idx (see combo_check_tensors).  A row of an [N][P] array is
 * one tensor; so is every layer's piece of it.
 *
 * combo_grad_norm writes norm_out and coef_out (device float[N]; either may be
 * NULL); combo_grad_clip writes them and the clipped tensors to the addresses in
 * d_out (as d_tensors; an output may be its input, and must not overlap any other
 * input).  A tensor that is its own output and whose coefficient is 1 is not
 * rewritten.  A norm that is infinite gives c = 0, one that is NaN gives NaN, and
 * the outputs follow by the formula; a worker without elements has norm 0.
 * max_norm >= 0.
 *
 * Arithmetic: squares are summed in binary32 over at most 16 elements and in
 * binary64 beyond (wholly in binary64 where the squares leave binary32's range),
 * in an order that depends on the sizes alone; out is the binary32 product,
 * rounded once.  scratch: device memory of at least combo_grad_scratch_bytes(N)
 * bytes, 8-byte aligned, contents undefined afterwards.  Two launches on
 * `stream`.  total < 2^46.
 */
size_t combo_grad_scratch_bytes(int N);
combo_status combo_grad_norm(const void* const* d_tensors, const int64_t* d_begin, const int32_t* d_first,
                             int n_tensors, int N, int64_t total, int elem_bytes, float max_norm,
                             float* norm_out, float* coef_out, void* scratch, size_t scratch_bytes,
                             void* stream);
combo_status combo_grad_clip(const void* const* d_tensors, void* const* d_out, const int64_t* d_begin,
                             const int32_t* d_first, int n_tensors, int N, int64_t total, int elem_bytes,
                             float max_norm, float* norm_out, float* coef_out, void* scratch,
                             size_t scratch_bytes, void* stream);

/* Debug helper for the two calls above: *dev_flag (device int32) becomes 0 when the
 * table is as described (ascending, ends in place, non-empty tensors non-null and
 * aligned), else 1 + a bad tensor, or 1 + n_tensors + a bad worker. */
combo_status combo_check_tensors(const void* const* d_tensors, const int64_t* d_begin, const int32_t* d_first,
                                 int n_tensors, int N, int64_t total, int elem_bytes, void* stream,
                                 int32_t* dev_flag);

/*
 * Group norm with an activation, channels last, for samples of all workers.  x is
 * [B][L][C] (B samples of L positions), `groups` groups of C / groups neighbouring
 * channels; w is the worker a sample belongs to:
 *
 *   mean, rstd = 1 / sqrt(var + eps) over a (sample, group),  var biased
 *   h = (x - mean) * rstd,   z = h * gamma_w + beta_w,   y = act(z)
 *
 * and backward, from dy and the mean and rstd the forward call wrote:
 *
 *   dz = dy * act'(z),   dgamma_w = sum dz * h,   dbeta_w = sum dz     (w's samples)
 *   t = dz * gamma_w,    dx = rstd * (t - mean(t) - h * mean(t * h))
 *
 * x, y, dy, dx: elem_bytes 4 = float or 2 = bfloat16, aligned to it; positions lie
 * `..._pitch` >= C elements apart, samples L pitches.  y may be x, and dx may be x or
 * dy, with the same pitch; other overlaps are refused (arrays of one pitch whose channels
 * lie beside each other, views of one wider array, do not overlap).  gamma, beta: param_bytes 4 or
 * 2, worker w's at + w * param_pitch elements -- a flat [N][P] array is given by its
 * first vector's place and pitch P --; both NULL for 1 and 0.  d_begin: device
 * int64[N + 1], worker w's samples are d_begin[w] .. d_begin[w+1] - 1 (ascending,
 * d_begin[0] = 0, d_begin[N] = B; trusted, like idx); NULL if N == 1.  A worker may
 * have no sample.  mean, rstd: float [B][groups], NULL in the forward call if not
 * wanted.  dgamma, dbeta: float, worker w's at + w * grad_pitch, written (not added
 * to), zeros for a worker without samples; both NULL if not wanted.
 *
 * Arithmetic: binary32, rounded once to bfloat16 at the end.  Statistics by merging
 * (count, mean, sum of squared deviations), so a large mean costs no more than its rounding to
 * binary32 does (two or three units of its last place).  z is formed
 * in the order written, without fused operations, in both calls: where ReLU clipped
 * (z <= 0), dz is 0 whatever dy holds.  ReLU keeps NaN; NaN and infinity stay in their
 * (sample, group).  SiLU and its slope are within six units of binary32's last place for
 * float arrays, of the sums they enter for slopes near 0; for bfloat16 arrays the exponential
 * in them errs by 2 + 1.2 |z| units, far below the result's rounding (0 where z < -87).
 * Results do not change from run to run.
 *
 * scratch (both calls): device memory of at least combo_group_norm_scratch_bytes bytes,
 * 16-byte aligned, contents undefined afterwards.
 * C / groups <= COMBO_NORM_MAX_CHANNELS, B * L * C <= 2^40.
 */
enum { COMBO_ACT_NONE = 0, COMBO_ACT_RELU = 1, COMBO_ACT_SILU = 2 /* z / (1 + exp(-z)) */ };
#define COMBO_NORM_MAX_CHANNELS 4096
combo_status combo_group_norm(const void* x, int64_t x_pitch, void* y, int64_t y_pitch, int elem_bytes,
                              const void* gamma, const void* beta, int param_bytes, int64_t param_pitch,
                              const int64_t* d_begin, int N, int64_t B, int64_t L, int64_t C, int groups,
                              float eps, int act, float* mean_out, float* rstd_out, void* scratch,
                              size_t scratch_bytes, void* stream);
size_t combo_group_norm_scratch_bytes(int64_t B, int64_t L, int64_t C, int groups);
combo_status combo_group_norm_backward(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch,
                                       void* dx, int64_t dx_pitch, int elem_bytes, const void* gamma,
                                       const void* beta, int param_bytes, int64_t param_pitch,
                                       const int64_t* d_begin, int N, int64_t B, int64_t L, int64_t C,
                                       int groups, int act, const float* mean, const float* rstd,
                                       float* dgamma, float* dbeta, int64_t grad_pitch, void* scratch,
                                       size_t scratch_bytes, void* stream);

/*
 * Products grouped by worker: every worker's rows (samples) times its own weights,
 * a layer without bias in one call for all workers, however many rows each has.
 *
 *   combo_grouped_linear              y[m][n]    = sum_k x[m][k] W_w[n][k]
 *   combo_grouped_linear_grad_input   dx[m][k]   = sum_n dy[m][n] W_w[n][k]
 *   combo_grouped_linear_grad_weight  dW_w[n][k] = sum_m dy[m][n] x[m][k]
 *
 * m runs over the M rows, worker w's being d_begin[w] .. d_begin[w+1] - 1 (device
 * int64[N + 1], ascending, within 0 .. M; trusted, like idx; rows of no worker are
 * neither read into a result nor written), k over n_in, n over n_out.  Rows of x, y,
 * dx, dy lie `..._pitch` elements apart.  W_w is at w + v * w_stride elements for
 * worker v, its rows w_pitch >= n_in apart: a layer inside a flat [N][P] array is given
 * by its first weight's place, pitch n_in and stride P.  The same holds for dW, which
 * is written (not added to), zeros for a worker without rows.
 *
 * elem_bytes (of the inputs) / out_bytes: 4 / 4 float; 2 / 2 and 2 / 4 bfloat16 in,
 * bfloat16 or float out.  float: multiply-adds in binary32, in the order of the sum, one
 * chain (off by 1e-6 of the result over 4096 terms of either sign, 9e-6 over 262144).
 * bfloat16: exact products, summed in binary32 by the tensor cores, which truncate at every
 * addition of 16 products: about 1e-6 of the sum of the magnitudes for sums over 1000, 8e-6 over
 * 4096; longer sums are cut into parts of 4096 that are added with rounding, so it stays at that.
 * The result is rounded once.  Outputs must not overlap inputs (rows of one pitch may lie
 * beside each other in a wider array).  A NaN or infinity reaches the results that
 * its row and its worker's weights enter, no others.  Results do not change from run to run.
 * Bases, pitches and strides that are all multiples of 16 bytes make large bfloat16 products
 * about ten times as fast as others; so a flat [N][P] array of bfloat16 wants a P and layers'
 * places that are multiples of 8.
 */
#define COMBO_LINEAR_MAX_WIDTH (1 << 20)   /* n_in, n_out */
#define COMBO_LINEAR_MAX_ROWS (1 << 22)    /* M */
combo_status combo_grouped_linear(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch,
                                  int64_t w_stride, void* y, int64_t y_pitch, int elem_bytes, int out_bytes,
                                  const int64_t* d_begin, int N, int64_t M, int64_t n_in, int64_t n_out,
                                  void* stream);
combo_status combo_grouped_linear_grad_input(const void* dy, int64_t dy_pitch, const void* w, int64_t w_pitch,
                                             int64_t w_stride, void* dx, int64_t dx_pitch, int elem_bytes,
                                             int out_bytes, const int64_t* d_begin, int N, int64_t M,
                                             int64_t n_in, int64_t n_out, void* stream);
combo_status combo_grouped_linear_grad_weight(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch,
                                              void* dw, int64_t dw_pitch, int64_t dw_stride, int elem_bytes,
                                              int out_bytes, const int64_t* d_begin, int N, int64_t M,
                                              int64_t n_in, int64_t n_out, void* stream);

/*
 * Softmax cross entropy of a linear classifier, grouped by worker: every worker's rows
 * against its own weights, the logits never kept.
 *
 *   z_mv = x_m . W_w,v      lse_m = log sum_v exp z_mv      loss_m = lse_m - z_m,label
 *
 * and the gradients of sum_m g_m loss_m:
 *
 *   d_mv = (exp(z_mv - lse_m) - [v = label_m]) g_m
 *   dx_m = sum_v d_mv W_w,v      dW_w,v = sum_m d_mv x_m
 *
 * x, w, d_begin and their pitches and strides: as combo_grouped_linear, n_out being the
 * number of classes.  d_labels: device int64[M]; a row whose label is not in
 * 0 .. n_out - 1 has none: its loss, lse and dx are 0, and whatever it holds (NaN too)
 * enters nothing.  Rows of no worker are neither read into a result nor written.
 * loss_out, lse_out: device float[M].  Backward takes the lse that the forward call wrote,
 * and row_grad, device float[M], the g_m; NULL stands for every worker's mean, g_m = 1 /
 * (labelled rows of m's worker).  dx [M][n_in] of x's type; dW as in
 * combo_grouped_linear_grad_weight, grad_bytes 4 = float or, for bfloat16 inputs, 2 =
 * bfloat16; written (not added to), zeros for a worker without labelled rows.
 *
 * Outputs must not overlap inputs, scratch or one another (x and dx may lie beside each
 * other in a wider array).  A NaN or infinity reaches the results that its row and its
 * worker's weights enter, no others.  Results do not change from run to run (with as much scratch).
 *
 * Arithmetic: logits, exponentials and sums in binary32, relative to the row's largest
 * logit; an exponential below 2^-126 counts as 0.  Losses and d are formed from
 * differences of logits: what that adds to the logits' own errors does not grow with their
 * size, and no loss is below 0.  A class at -inf has probability 0
 * (bfloat16; an infinite float may make its logits NaN).  The classes are taken a piece
 * at a time, in backward with d in scratch between the products that form it and those
 * that use it.
 * bfloat16: exact products, summed as in combo_grouped_linear, in parts of 1024 (a float
 * dW: of 256; up to 256 classes of 128, its logits of 256) added with rounding.  d is rounded to bfloat16 once for dx (what
 * that leaves of the label's d, most of a row's gradient, is added in binary32) and for a
 * bfloat16 dW of more than 128 rows a worker on average; a bfloat16 dW of fewer takes 16
 * bits of it, a float dW 24.  With row_grad NULL the mean's factor is applied behind the
 * products.
 * float: products of parts of 22 bits (forward; 2^-39 of the row's or class's largest value
 * where that is more) and 24 bits (backward), relative errors of some 1e-7 to 5e-7 of the
 * sums' magnitudes; small problems by multiply-adds.
 * bfloat16 weights whose base, pitch and stride are multiples of 16 bytes are read where
 * they lie; others, and floats, are brought into scratch a piece at a time.
 *
 * scratch: device memory, 256-byte aligned, contents undefined afterwards, of
 * combo_grouped_cross_entropy_scratch_bytes bytes (grad_bytes 0 for the forward call), or
 * of less, down to combo_grouped_cross_entropy_least_scratch_bytes: the classes are then
 * taken in smaller pieces, at the price of time and, in backward, of another order in
 * which dx is added up.  With R = M + 63 min(N, M) (every worker's rows are rounded up to
 * 64, labelled or not), K = n_in up to a multiple of 128 and V = n_out it holds, in bytes,
 *   packed rows           2 R K (bfloat16), 4 R K (floats, forward), 6 R K (backward)
 *   forward               R V / 16 to R V / 4 of pieces' maxima and sums
 *   backward              4 R K of dx's sums, more where they are cut into parts
 *   a piece of C classes  2 R C or 4 R C of d (bfloat16 dW), 6 R C (float), and the weights' parts:
 *                         2 N C K (bfloat16 off 16 bytes), 4 N C K (floats, forward), 6 N C K
 * with C from 128 or 256, or all there are if that is less, up to what 640 MB hold.
 * A forward call on bfloat16 weights on 16 bytes has no pieces: it is as fast with the
 * least.  Few rows and classes (multiply-adds): 4 M n_out bytes in backward.
 */
size_t combo_grouped_cross_entropy_scratch_bytes(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes,
                                                 int grad_bytes);
size_t combo_grouped_cross_entropy_least_scratch_bytes(int N, int64_t M, int64_t n_in, int64_t n_out, int elem_bytes,
                                                       int grad_bytes);
combo_status combo_grouped_cross_entropy(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch,
                                         int64_t w_stride, int elem_bytes, const int64_t* d_labels,
                                         const int64_t* d_begin, int N, int64_t M, int64_t n_in, int64_t n_out,
                                         float* loss_out, float* lse_out, void* scratch, size_t scratch_bytes,
                                         void* stream);
combo_status combo_grouped_cross_entropy_backward(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch,
                                                  int64_t w_stride, int elem_bytes, const int64_t* d_labels,
                                                  const float* lse, const float* row_grad, void* dx,
                                                  int64_t dx_pitch, void* dw, int64_t dw_pitch, int64_t dw_stride,
                                                  int grad_bytes, const int64_t* d_begin, int N, int64_t M,
                                                  int64_t n_in, int64_t n_out, void* scratch,
                                                  size_t scratch_bytes, void* stream);

/*
 * Dropout whose mask is a function of counters and is never stored:
 *
 *   y = residual + (kept ? x * 65536 / (65536 - T) : 0),   T = p * 65536 rounded
 *
 * x, residual (NULL: none), y: [M][n], elem_bytes 4 = float or 2 = bfloat16, rows
 * `..._pitch` >= n elements apart, worker w's being d_begin[w] .. d_begin[w+1] - 1 (as
 * above; NULL if N == 1: all rows).  The backward pass is the same call on dy without a
 * residual.
 *
 * kept: with `step` one step of splitmix64 (the output for state z), worker
 * W = first_worker + w, the element's row r among its worker's and column c,
 *
 *   key = step(step(step(seed) ^ (round << 32 | W)) ^ (2^63 | site))
 *   h = step(key ^ (r * ceil(n / 4) + c / 4)),   kept = (h >> 16 (c % 4)) % 65536 >= T
 *
 * so a worker's mask is the same whichever other workers are in the call and whichever GPU
 * holds it; `site` tells apart the dropouts of one step.  p in 0 .. 1; p = 1 keeps nothing.
 * Dropped elements are 0 (or the residual) whatever x holds.  binary32 product and sum, each
 * rounded; rounded once more to bfloat16.  y may be x or residual (same pitch); other
 * overlaps with y, d_begin's too, are refused.  n <= 2^32, M * n <= 2^40, first_worker + N <=
 * COMBO_MAX_WORKERS.
 */
combo_status combo_dropout(const void* x, int64_t x_pitch, const void* residual, int64_t residual_pitch, void* y,
                           int64_t y_pitch, int elem_bytes, const int64_t* d_begin, int N, int64_t M, int64_t n,
                           float p, uint64_t seed, uint32_t round, uint32_t site, int first_worker, void* stream);

/*
 * Reads and clears the device status word that kernels set when one of their
 * bounded waits gives up.  Synchronises the device.  Returns COMBO_OK or
 * COMBO_ERR_DEVICE_TIMEOUT (or COMBO_ERR_CUDA).
 */
combo_status combo_device_status(void);

/* Which aggregation kernel the last combo_segment_aggregate* call on this
 * thread launched: 0 none, 1 direct gather, 2 shared-memory staged (persistent
 * CTAs, a ring of tiles), 3 row pull, 5 shared-memory staged with one tile per
 * CTA (short inputs). */
int combo_last_kernel_path(void);

/* Which kernels the last combo_grouped_linear*, combo_grouped_cross_entropy* or
 * combo_group_norm* call on this thread launched: 0 none; products and cross entropy:
 * 1 multiply-adds (products of floats, small cross entropies), 2 tensor cores, one CTA
 * a tile, 3 tensor cores, a pair of CTAs a tile, 4 tensor cores, operands brought by
 * threads (bases, pitches or strides off 16 bytes); group norm: 5 slabs resident in
 * shared memory, 6 streamed in two passes. */
int combo_last_step_path(void);

/* Forces a path for the following calls on this thread: 0 automatic (default),
 * 1 direct gather (blocks taken worker-fastest, so that the gather's re-reads
 * are served by L2), 2 staged with persistent CTAs (falls back to direct where
 * staging cannot apply), 5 staged with one tile per CTA (falls back to 2 where
 * rows differ in their 16-byte phase or a tile does not fit), 6 direct gather
 * in the naive order, row after row (the contrast case for profiling: its
 * re-reads mostly come from DRAM); with combo_segment_aggregate_rows: 3 nothing
 * staged. */
void combo_set_kernel_path(int path);

/* Expert knob for the staged kernel, this thread only: tile width in elements
 * (a multiple of 256 up to 2048; for rows whose byte pitch is not a multiple
 * of 16 every 256 asked for become 256 - 16/elem_bytes) and number of pipeline
 * stages; 0 = chosen automatically.  A tile that cannot be honoured makes
 * the call fall back to the direct kernel.  combo_segment_aggregate_rows takes
 * the widest 256 * 2^k columns that do not exceed the tile asked for, and at
 * least three stages. */
void combo_set_tuning(int tile_elems, int stages);

/* This thread only: whether the staged aggregation kernel is launched with
 * programmatic stream serialization (default 1).  With it the kernel may be
 * scheduled while the preceding kernel of the same stream is still draining;
 * it waits for that kernel to complete before its first access to global
 * memory, so stream order as seen through memory is unchanged.  What it
 * hides is launch latency and set-up between back-to-back rounds (Section
 * 4.1: one synchronization per iteration).  0 = ordinary launches. */
void combo_set_launch_overlap(int on);

/* Widest column range a single aggregation launch takes (the staged kernels
 * address columns with signed 32-bit copy coordinates).  Wider inputs are cut
 * into column shards of this many columns inside the call, one launch each;
 * Eq. 3 couples workers only at equal column, so the result is the same. */
int64_t combo_max_launch_columns(void);

/* Expert / test knob, this thread only: cut inputs into shards of `columns`
 * columns instead (rounded down to a multiple of 64; 0 or out of range
 * restores combo_max_launch_columns()). */
void combo_set_launch_columns(int64_t columns);

/*
 * Self-check of the time-out path (no counterpart in the paper).  Every wait
 * inside the kernels is bounded; a wait that runs out sets the device status
 * word and the kernel returns, which combo_device_status() then reports as
 * COMBO_ERR_DEVICE_TIMEOUT.  This call enqueues a one-warp kernel that waits,
 * with a cap of a thousand polls, on a barrier of its own that nothing ever
 * signals, and reports in the same way: after it, combo_device_status()
 * returns COMBO_ERR_DEVICE_TIMEOUT once (site 99 in combo_last_cuda_error())
 * and COMBO_OK afterwards.  It touches no product kernel and leaves nothing
 * armed; the device and the context stay usable.
 */
combo_status combo_debug_dead_wait(void* stream);

const char* combo_status_string(combo_status status);
const char* combo_last_cuda_error(void);
int combo_version(void);

#ifdef __cplusplus
}
#endif
#endif /* COMBO_B200_H */
