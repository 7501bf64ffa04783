/*
 * pnn.h -- C ABI of the MI355X (gfx950) parallel neural network (PNN) library.
 *
 * The method (Kalwarowskyj & Schikuta, "Parallel Neural Networks in Golang", section
 * "Parallel Neuronal Networks"): the training set is split into K slices; K child networks
 * (CNs), all started from one parameter vector, each train on their own slice with
 * back-propagation and (mini-batch) stochastic gradient descent (section "Fundamentals",
 * eq. (2)-(13)); the CNs are then combined into one network by averaging all weights and
 * all biases.  One handle serves a single sequential network (K = 1) and a PNN (K > 1)
 * alike, as the paper's TrainableNetwork interface does (section "Implementation Details").
 *
 * Conventions shared by every call:
 *  - Device pointers (suffix _dev) are HIP device memory owned by the caller; the library
 *    never frees them and does not keep them after the call returns.
 *  - The library owns the parameters and its workspace (allocated in pnn_init, released
 *    in pnn_destroy).
 *  - `hip_stream` is a hipStream_t (NULL = the default stream).  Device work is enqueued on
 *    it and the call returns once enqueued; only pnn_get_params, pnn_set_params, pnn_eval
 *    and a pnn_infer call with correct_host != NULL wait for the device.  After a training
 *    epoch on a persistent plan (pnn_plan), the next call that consumes the CNs other than
 *    pnn_train_epoch first waits for that epoch to end, to read its failure flag.
 *  - pnn_train_epoch, pnn_train_epoch_order, pnn_merge, pnn_infer (without a count), pnn_infer_routed
 *    and pnn_train_routed may be recorded into a graph, after a call of the same kind with at least as many rows has sized the
 *    handle's workspace (growth is refused while the stream records: PNN_EHIP, nothing recorded).  The
 *    graph may be replayed until pnn_destroy, also after later calls with more rows.
 *  - Errors are returned as a pnn_status; the message of the last failure is available
 *    from pnn_last_error (per handle; a NULL handle gives the message of the last failed
 *    pnn_init, or other call without a handle, on the calling thread).  No exception or abort
 *    crosses the interface.
 *  - One handle must not be used from two host threads at once.
 *  - Input rows x_dev are read with 16-byte vector loads: x_dev must be 16-byte aligned
 *    (PNN_EINVAL otherwise); sizes[0] is a multiple of 8, so every row then is too.
 *
 * Parameter layout (host side, get/set): one network is P = pnn_param_count(cfg) floats,
 * W1, b1, W2, b2, ..., W_l row-major [sizes[l]][sizes[l-1]], b_l [sizes[l]].
 */
#ifndef PNN_H
#define PNN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pnn_net pnn_net; /* opaque, library-owned */

typedef enum {
    PNN_OK = 0,
    PNN_EINVAL = -1, /* invalid configuration or argument (NULL pointer, bad index) */
    PNN_ESHAPE = -2, /* sizes do not fit (N < K leaves a slice empty, n < 0, ...) */
    PNN_ENOMEM = -3, /* device allocation failed */
    PNN_EHIP = -4,   /* a HIP runtime call or kernel launch failed */
    PNN_ESTATE = -5  /* the handle is unusable after an earlier device failure */
} pnn_status;

/* Activation of a layer.  Rectifier eq. (4), softmax eq. (5); sigmoid and tanh are named in
 * section "Activation Functions in Single- and Parallel Neuronal Networks" (textbook forms);
 * leaky rectifier with slope 0.01 for z < 0.  The rectifier's derivative at z = 0 is 1
 * (eq. (4) puts z = 0 in the linear branch).  Softmax is allowed on the output layer only. */
typedef enum { PNN_SIGMOID = 0, PNN_TANH = 1, PNN_RELU = 2, PNN_LEAKY_RELU = 3, PNN_SOFTMAX = 4 } pnn_act;

/* Output error rule.  MSE: quadratic cost 1/2 sum (x - e)^2 with eq. (9),
 * delta^L = (x^L - e) (.) phi'(z^L).  XENT: eq. (10), delta^L = x^L - e, for a softmax
 * output (eq. (6) cost) or a sigmoid output (binary cross-entropy). */
typedef enum { PNN_LOSS_MSE = 0, PNN_LOSS_XENT = 1 } pnn_loss;

/* FP32: every value stored in fp32.  BF16_MIXED: inputs, hidden activations, weights and
 * deltas enter the matrix products as bfloat16 (round to nearest even) with fp32
 * accumulation; biases, activations' arithmetic, softmax and the master weights are fp32. */
typedef enum { PNN_FP32 = 0, PNN_BF16_MIXED = 1 } pnn_precision;

typedef struct {
    int32_t n_layers;  /* L weight layers, 1..8 */
    int32_t sizes[9];  /* sizes[0] inputs ... sizes[L] outputs (classes), each >= 1 */
    int32_t act[8];    /* pnn_act of weight layer l+1 */
    int32_t loss;      /* pnn_loss */
    int32_t precision; /* pnn_precision */
    int32_t replicas;  /* K >= 1 child networks */
    int32_t batch;     /* B >= 1; 1 = per-sample stochastic gradient descent */
    float lr;          /* eta, eq. (12)-(13) */
} pnn_config;

/* Checks a configuration without touching the GPU.  Rules: 1 <= L <= 8; sizes >= 1 and
 * sizes[l] % 8 == 0 for every layer except the output layer, whose width is <= 16;
 * softmax only on the output layer and only with PNN_LOSS_XENT; XENT needs a sigmoid or
 * softmax output; K >= 1, B >= 1, finite lr >= 0.  Returns PNN_OK or PNN_EINVAL. */
pnn_status pnn_config_check(const pnn_config* cfg);

/* P, the number of parameters of one network: every weight W_kj and every bias b_k of each
 * layer (eq. (2): sizes[l] * sizes[l-1] weights and sizes[l] biases per layer l), which is what
 * the combination averages (section "Implementation Details").  0 for an invalid
 * configuration. */
int64_t pnn_param_count(const pnn_config* cfg);

/* Dataset split (section "Implementation Details": the dataset is split according to the
 * number of CNs): slice k of N samples over K CNs is the contiguous row range
 * [start, start + len); the first N mod K slices hold one more sample.  Host only. */
pnn_status pnn_shard(int64_t N, int32_t K, int32_t k, int64_t* start, int64_t* len);

/* Creates a handle on the current HIP device.  theta0_host (P floats, host memory, read
 * during the call) is cloned into all K child networks and into the merged network
 * (section "Accuracy and Confidence of Networks": the PNN's CNs start as clones of one
 * random network).  *out receives the handle; NULL on failure. */
pnn_status pnn_init(const pnn_config* cfg, const float* theta0_host, void* hip_stream, pnn_net** out);

/* One training epoch of every CN over its own slice (sections "Gradient Descent" and
 * "Implementation Details").  x_dev: [N][sizes[0]] row-major fp32; y_dev: [N] int32
 * class labels in [0, sizes[L]).  CN k visits rows of its slice in ascending order in
 * batches of B (the last batch may be shorter); each batch's gradients are averaged before
 * the update W <- W - eta / B_t * sum_b delta_b x_b^T, b <- b - eta / B_t * sum_b delta_b.
 * Requires N >= K (PNN_ESHAPE otherwise).  Labels outside [0, sizes[L]) give an undefined
 * (but memory-safe) update. */
pnn_status pnn_train_epoch(pnn_net* net, const float* x_dev, const int32_t* y_dev, int64_t N, void* hip_stream);

/* One epoch over the rows in a given order (the per-epoch shuffling that the paper leaves
 * open: it trains on the slices in their stored order).  Equivalent to pnn_train_epoch on
 * x[order[0..N)], y[order[0..N)]: epoch row r is data-set row order_dev[r], and the K slices
 * are the contiguous ranges of that sequence.  order_dev [N] int32 on the device, normally a
 * permutation drawn by the caller from a seeded generator (within each slice's range for a
 * per-CN shuffle); entries outside [0, N) select row 0.  The rows are gathered into a
 * library-owned staging copy (N x sizes[0] floats, grown with hipMalloc when a larger N
 * arrives) on the caller's stream.  Errors as pnn_train_epoch; N must fit int32. */
pnn_status pnn_train_epoch_order(pnn_net* net, const float* x_dev, const int32_t* y_dev, int64_t N,
                                 const int32_t* order_dev, void* hip_stream);

/* Combination by averaging (section "Implementation Details"): merged := (1/K) sum_k theta_k
 * for every weight and bias, accumulated in fp64 with k ascending, rounded once to fp32.
 * broadcast != 0 also copies the merged network back into every CN (model averaging
 * between epochs); with the fused last-layer plan (pnn_plan) that copy is made by the next
 * epoch's first step, which reads the merged network, or on demand by the first other call
 * that reads a CN's parameters: every call sees the CNs as copied. */
pnn_status pnn_merge(pnn_net* net, int32_t broadcast, void* hip_stream);

/* Weighted combination: the paper notes that CNs can be combined in several ways and leaves
 * better combination functions to future work (sections "Parallel Neuronal Networks" and
 * "Findings and Conclusion") without defining one; this one is the weighted mean:
 * merged := sum_k w_k theta_k / sum_k w_k, each product and the sum in fp64 with k ascending,
 * rounded once to fp32.  weights_host: K host doubles, each finite and >= 0, with a positive sum
 * (PNN_EINVAL otherwise, nothing launched).  Equal weights give pnn_merge's result bitwise.
 * broadcast as in pnn_merge.  The weights are copied to a library-owned device array before
 * the call returns (the call waits for the stream's earlier work). */
pnn_status pnn_merge_weighted(pnn_net* net, const double* weights_host, int32_t broadcast, void* hip_stream);

/* Classification (sections "Fundamentals" and "MNIST Dataset": one output neuron per class,
 * tested on unseen data).  which = -1 uses the merged network, 0..K-1 one CN.
 * x_dev [n][sizes[0]] fp32.  pred_dev [n] int32 receives the argmax of the outputs (lowest
 * index on ties).  out_dev (nullable) [n][sizes[L]] fp32 receives the outputs x^L.  When
 * y_dev [n] and correct_host are both non-NULL, the call waits for the device and writes
 * the number of rows with pred == y to *correct_host.  n = 0 reads and writes nothing on the
 * device (the pointers may be NULL) and sets *correct_host, if given, to 0. */
pnn_status pnn_infer(pnn_net* net, int32_t which, const float* x_dev, int64_t n, int32_t* pred_dev, float* out_dev,
                     int64_t* correct_host, const int32_t* y_dev, void* hip_stream);

/* Evaluation of one network on labelled rows: the accuracy test of the merged network
 * (sections "Implementation Details" and "MNIST Dataset") and the per-CN comparison and cost
 * per epoch of the experiments.  which = -1 merged, 0..K-1 one CN.  x_dev [n][sizes[0]] fp32
 * and y_dev [n] int32 are the caller's device arrays (labels in [0, sizes[L])).  Writes
 *   *correct_host (nullable): rows whose argmax output (lowest index on ties) equals the label;
 *   *cost_host (nullable): the mean cost over the rows, the cost whose output error training
 *     uses: quadratic 1/2 sum_o (x_o - e_o)^2, or with PNN_LOSS_XENT the cross-entropy
 *     (-log x_label for a softmax output, eq. (6); -sum_o [e_o log x_o + (1 - e_o) log(1 - x_o)]
 *     for a sigmoid output), each row's cost in fp64 from the fp32 outputs, the rows summed in
 *     a fixed order in fp64.
 * Waits for the device.  The library owns a per-row cost buffer of the largest n seen (grown
 * with hipMalloc on the first call that needs more).  n = 0 gives 0 and 0.0 without device work;
 * a NULL x_dev or y_dev is PNN_EINVAL. */
pnn_status pnn_eval(pnn_net* net, int32_t which, const float* x_dev, const int32_t* y_dev, int64_t n,
                    int64_t* correct_host, double* cost_host, void* hip_stream);

/* pnn_eval without any device allocation, for callers that cannot allocate device memory
 * (code that must not call hipMalloc: tight evaluation loops in serving or training, harnesses
 * that forbid allocation).  Same arguments, results and errors as pnn_eval, computed by the same
 * kernels; its workspace (a count, a sum, one 8,192-row chunk's hidden activations and, when
 * cost_host is given, n per-row costs) lives in a fixed 64 MiB device array that the library
 * holds on every GPU it runs on until the process ends, instead of in buffers grown with
 * hipMalloc.  A call that needs more workspace than that returns PNN_ESHAPE and launches
 * nothing (with cost_host: n <= 8,388,576 - 1,024 A up to alignment, A the bytes of hidden
 * activations of one row: 4 per hidden neuron, 2 in bf16-mixed precision).  Every call on one GPU shares that GPU's array, which keeps the last call's contents:
 * calls that overlap in time on one GPU (other host threads, other streams) race and must be
 * serialised by the caller. */
pnn_status pnn_eval_noalloc(pnn_net* net, int32_t which, const float* x_dev, const int32_t* y_dev, int64_t n,
                            int64_t* correct_host, double* cost_host, void* hip_stream);

/* Copies one network's parameters (which = -1 merged, 0..K-1 a CN) to host_out (P floats)
 * in the layout above.  Waits for the device. */
pnn_status pnn_get_params(pnn_net* net, int32_t which, float* host_out);

/* Overwrites parameters from host_in (P floats): which = -1 the merged network, 0..K-1 one
 * CN, -2 every CN and the merged network.  Waits for the device.  Used for checkpoint and
 * resume: training continued from restored parameters is bitwise identical. */
pnn_status pnn_set_params(pnn_net* net, int32_t which, const float* host_in);

/* Message of the last failure on this handle ("" if none); NULL net: last failure of pnn_init, or
 * of another call without a handle, on the calling thread.  The string lives until the next call on
 * the same handle. */
const char* pnn_last_error(const pnn_net* net);

/* Device time of the library's kernels, for throughput accounting.  pnn_profile(net, 1)
 * starts recording a HIP event pair around every kernel the library launches (this adds
 * host overhead; leave it off when measuring whole-call throughput) and clears the
 * counters; pnn_profile(net, 0) stops.  pnn_profile_read fills up to `cap` entries of
 * names (static strings), total_ms and launches, waits for the device, and returns the
 * number of distinct kernels recorded. */
pnn_status pnn_profile(pnn_net* net, int32_t enable);
int32_t pnn_profile_read(pnn_net* net, const char** names, double* total_ms, int64_t* launches, int32_t cap);

/* Name of the training plan that pnn_init chose for the handle (a static string; "" for
 * a NULL handle).  All plans compute the update of pnn_train_epoch and differ only in the
 * order of fp32 roundings:
 *  "per-sample persistent"  fp32, B = 1, one hidden layer, sizes[0] <= 832: one launch per epoch
 *                           for each group of CNs whose workgroups fit the device at once.  Any
 *                           number of CNs up to 128 neurons; up to 384 neurons and 256 CNs, where
 *                           long slices are the faster for it (few groups).  Above 128 neurons an
 *                           epoch of short slices, or one that is recorded into a graph, runs as in
 *                           the chunked plan;
 *  "per-sample chunked"     fp32, B = 1, one hidden layer of <= 1,024 neurons otherwise: kernel
 *                           launches per chunk of steps, for all CNs at once;
 *  "mini-batch persistent"  one hidden layer of <= 512 neurons, <= 16 outputs, sizes[0] % 16 == 0
 *                           and <= 832: one launch per epoch for each group of CNs whose
 *                           ceil(H / 16) (or ceil(H / 32)) tile workgroups fit the device at once.
 *                           fp32, 2 <= B <= 32; and fp32 with 33 <= B <= 64 or bf16-mixed with
 *                           B <= 64, where that is the faster way (few groups or wide inputs).  An
 *                           epoch that is recorded into a graph runs as in "mini-batch";
 *  "mini-batch fused last layer"  fp32, one hidden layer of >= 256 neurons (a multiple of
 *                           4), B = 128, <= 16 outputs, sizes[0] >= 128 (a multiple of 4),
 *                           the split-bf16 products (not PNN_GEMM=fp32): kernel launches per
 *                           batch step, with the last layer's forward in the hidden layer's
 *                           forward and its hidden errors and update in the hidden layer's
 *                           update (one pass less over the hidden activations);
 *  "mini-batch"             otherwise: kernel launches per layer and batch step.
 * The environment variable PNN_MB_PLAN=launch, read by pnn_init, selects "mini-batch"
 * where "mini-batch persistent" or "mini-batch fused last layer" would apply.  The persistent
 * plans' workgroups wait for each other with bounded polls (PNN_SPIN_LIMIT, read by pnn_init, default 4194304 polls); a launch
 * that runs into the bound ends every workgroup and leaves the CNs' parameters unspecified.
 * The next call that consumes the CNs -- pnn_merge, pnn_merge_weighted, pnn_infer, pnn_eval,
 * pnn_get_params, pnn_set_params (each waits for the last persistent launch to end first) or
 * pnn_train_epoch (which does not wait: it sees the failure once that launch has ended, and a
 * persistent launch enqueued after the failed one ends at once) -- returns PNN_EHIP and marks
 * the handle unusable (PNN_ESTATE from then on).  PNN_TEST_STALL_WAITS=1 (tests of that path
 * only) makes the persistent kernels' waits run into the bound.  PNN_TEST_TILE_DELAY=n (n sleeps
 * of about 3 us, ordering tests only) starts half of every CN's tile workgroups late in the
 * per-sample persistent kernel; the results stay within rounding of an undelayed run. */
const char* pnn_plan(const pnn_net* net);

/* Releases the handle and everything it owns (NULL is ignored). */
void pnn_destroy(pnn_net* net);

/* ---------------------------------------------------------------------------------------------
 * Rows that name their network.  The calls above give every network a contiguous slice of the
 * rows, or all of them; here each row names the networks that it goes through, for any number of
 * rows per network.  These calls take no handle: every matrix, the plan and the workspaces are the
 * caller's device memory, nothing is kept between calls, and two calls may run at the same time if
 * they write to different memory.  All of them may be recorded into a graph.  Work runs on
 * hip_stream and on its device (the null stream: on the current device).  A row's values are
 * contiguous; `_ld` is the distance between rows and `_net` between networks, in values.  Rows need
 * be aligned to their type only (16-byte alignment and widths that are multiples of 8 are faster).
 * `type` is PNN_FP32 (fp32) or PNN_BF16_MIXED (bfloat16).  Products are summed in fp32.  fp32
 * operands enter the matrix units in three bf16 parts (six products, as exact as fp32 products), or
 * as they are in a forward product or an input gradient of at most 16 pairs a network in the mean.
 * So they have to be finite and below 3.38e38: an infinite operand makes what it reaches NaN where
 * it is taken in parts, and what fp32 arithmetic gives (infinite or NaN) where it is not; which of
 * the two depends on the number of pairs.  Parts end at 2^-133, so that operands below 2^-110 lose
 * their last bits.  Results must not overlap operands, and a plan is used with the sizes it was made
 * with.  What does not fit a launch (a result of more than 2^32 values of narrow rows, say) is refused
 * with PNN_ESHAPE. */

/* Row r's per_row ids are ids_dev[r per_row + j]: pair p = r per_row + j goes through network
 * ids_dev[p] in [0, networks); any other id drops the pair.  The same network may stand twice. */
typedef struct {
    const void* plan_dev; /* written by pnn_group_rows */
    int64_t n;            /* rows, n per_row <= 2^30 */
    int32_t per_row;      /* >= 1 */
    int32_t networks;     /* 1..1024 */
} pnn_groups;

/* Size of the plan of a grouping. */
pnn_status pnn_group_bytes(int64_t n, int32_t per_row, int32_t networks, int64_t* bytes);

/* Groups the pairs by network: a stable counting sort.  plan_dev (plan_bytes of memory, 16-byte
 * aligned) then holds, as int32: offsets[networks + 1], from the next multiple of four words on the
 * pair numbers: positions offsets[e] .. offsets[e + 1) are network e's pairs in ascending order, and
 * those from offsets[networks] on the dropped ones; then the library's own tables. */
pnn_status pnn_group_rows(const int32_t* ids_dev, int64_t n, int32_t per_row, int32_t networks, void* plan_dev,
                          int64_t plan_bytes, void* hip_stream);

/* One layer of every network: weights w_dev[e w_net + o w_ld + i], biases b_dev[e b_net + o] (fp32,
 * NULL for none).  A weight gradient reads the sizes and the type alone. */
typedef struct {
    int32_t inputs, outputs; /* 1..2^20 each */
    int32_t type;            /* of the weights, and of x, dy and a */
    const void* w_dev;
    int64_t w_net, w_ld;
    const float* b_dev;
    int64_t b_net;
} pnn_group_layer;

/* y[p] = phi(W_e x[p / per_row] + b_e) for every pair p of network e (eq. (2)-(3)); 0 for a dropped
 * pair.  act is an elementwise pnn_act or -1 for none.  x_dev [n][inputs], y_dev [n per_row][outputs]
 * of y_type. */
pnn_status pnn_grouped_forward(const pnn_groups* groups, const pnn_group_layer* layer, const void* x_dev, int64_t x_ld,
                               int32_t act, void* y_dev, int64_t y_ld, int32_t y_type, void* hip_stream);

/* Workspace of the two gradients below (0 where none is needed; either pointer may be NULL). */
pnn_status pnn_grouped_workspace(const pnn_groups* groups, const pnn_group_layer* layer, int64_t* input_bytes,
                                 int64_t* weights_bytes);

/* Hidden errors (eq. (11)): dx[r] = (sum_j W_e^T dy[r per_row + j]) (.) phi'(a[r]), the sum over the
 * row's pairs that are not dropped, j ascending; a row without one gets 0.  dy_dev [n per_row][outputs],
 * dx_dev [n][inputs] of dx_type.  act -1: no phi'; else a_dev [n][inputs] holds the stored activations
 * that the slope is read from (the rectifiers' derivative is 1 unless the sign bit is set). */
pnn_status pnn_grouped_backward_input(const pnn_groups* groups, const pnn_group_layer* layer, const void* dy_dev, int64_t dy_ld,
                                      const void* a_dev, int64_t a_ld, int32_t act, void* dx_dev, int64_t dx_ld,
                                      int32_t dx_type, void* ws_dev, int64_t ws_bytes, void* hip_stream);

/* Gradients of the weights and biases (eq. (12)-(13)): dw_e = sum_p dy[p] x[p / per_row]^T and
 * db_e = sum_p dy[p] over network e's pairs, in fp32; 0 for a network without pairs.  db_dev may be
 * NULL.  The sums' order depends on the sizes alone: the same call gives the same bits. */
pnn_status pnn_grouped_backward_weights(const pnn_groups* groups, const pnn_group_layer* layer, const void* dy_dev,
                                        int64_t dy_ld, const void* x_dev, int64_t x_ld, float* dw_dev, int64_t dw_net,
                                        int64_t dw_ld, float* db_dev, int64_t db_net, void* ws_dev, int64_t ws_bytes,
                                        void* hip_stream);

/* The forward product from 8-bit codes, for serving: rows and weights are integers in -127..127 with a scale
 * for each row and for each output of a network, a quarter of fp32's bytes and twice the rate of bf16. */

/* q[r][i] = the integer nearest to 127 x[r][i] / max_i |x[r][i]| (ties to even), scale[r] = max_i |x[r][i]| / 127
 * (fp32), so that x is about scale q.  x_dev [n][width] of `type`; q_dev int8 [n][width rounded up to a multiple of
 * 16], zeros past the width, its rows at multiples of 16 bytes.  A row of zeros has codes and a scale of 0, one
 * with a NaN or an infinity codes of 0 and a scale of NaN, which its products show. */
pnn_status pnn_quantize_rows(const void* x_dev, int64_t x_ld, int32_t type, int64_t n, int32_t width, int8_t* q_dev, int64_t q_ld,
                             float* scale_dev, void* hip_stream);

/* One layer of every network in codes: w_dev[e w_net + o w_ld + i] with scale_dev[e scale_net + o] (fp32), biases
 * as above.  inputs is a multiple of 16, at most 2^17 (sums are 32-bit integers and do not overflow); w_ld and w_net are
 * multiples of 16, w_dev is 16-byte aligned. */
typedef struct {
    int32_t inputs, outputs;
    const int8_t* w_dev;
    int64_t w_net, w_ld;
    const float* scale_dev;
    int64_t scale_net;
    const float* b_dev;
    int64_t b_net;
} pnn_group_codes;

/* y[p] = phi(x_scale[r] w_scale[e][o] sum_i x[r][i] w_e[o][i] + b_e), r = p / per_row, as pnn_grouped_forward; the sum
 * is exact, and rounded to fp32 once.  x_dev int8 [n][inputs], rows at multiples of 16 bytes; x_scale_dev [n]. */
pnn_status pnn_grouped_forward_int8(const pnn_groups* groups, const pnn_group_codes* layer, const int8_t* x_dev, int64_t x_ld,
                                    const float* x_scale_dev, int32_t act, void* y_dev, int64_t y_ld, int32_t y_type, void* hip_stream);

/* ---------------------------------------------------------------------------------------------
 * Rows that choose their networks.  A router scores every network for a row; the row goes through
 * the ones that it likes best, and their results are weighed into one.  No handle and nothing kept, as
 * for the grouped products above, whose ids these are.
 *
 * Row r has scores s [networks] of `type` and, with p = softmax(s), goes through the networks of its
 * per_row largest scores: ids, in descending order (lowest index on ties), and gates p at these, or
 * with `normalize` p divided by its sum over them.  A score of -inf is never chosen: a row with fewer
 * others has ids of -1 and gates of 0 at its end, and one of -inf alone takes no part.  A row with a
 * NaN or an infinite score has ids of -1 and gates, gradients and a balance loss of NaN.
 * With counts_e the pairs of network e, C their sum and n' the rows that take part, the balance loss is
 *   loss = networks sum_e (counts_e / C) (sum_r p_re) / n'
 * (1 where rows are spread evenly, 0 without rows).  Statistics and sums are fp32 (counts int32), and their order
 * depends on the sizes alone. */
typedef struct {
    const void* s_dev; /* [n][networks] */
    int64_t s_ld;
    int32_t type;
    int32_t networks;  /* 1..1024 */
    int64_t n;         /* < 2^31, n per_row <= 2^30 */
    int32_t per_row;   /* 1..64, <= networks */
    int32_t normalize;
} pnn_router;

/* Workspace of a pnn_route that counts. */
pnn_status pnn_route_bytes(int64_t n, int32_t networks, int64_t* bytes);

/* ids_dev int32 [n][per_row], gates_dev fp32 [n][per_row]; counts_dev int32 [networks + 1] (the pairs of
 * each network, then n') and loss_dev fp32 [1], or neither (and then no workspace). */
pnn_status pnn_route(const pnn_router* args, int32_t* ids_dev, float* gates_dev, int32_t* counts_dev, float* loss_dev,
                     void* ws_dev, int64_t ws_bytes, void* hip_stream);

/* ds_dev [n][networks] of `type`: the gradient of the scores from dgates_dev fp32 [n][per_row] (nullable)
 * at the chosen ids, pnn_route's or others (what stands at an id outside the networks is not read), and from dloss_dev fp32 [1]
 * (nullable), the balance loss's (counts_dev; the counts themselves have no gradient).  ds_dev may be
 * s_dev (with the same distance between rows). */
pnn_status pnn_route_grad(const pnn_router* args, const int32_t* ids_dev, const int32_t* counts_dev, const float* dgates_dev,
                          const float* dloss_dev, void* ds_dev, int64_t ds_ld, void* hip_stream);

/* Results of pairs, weighed into rows: out[r] = sum_j w[r per_row + j] y[r per_row + j], j ascending, over
 * the pairs whose id lies in [0, networks); 0 without one.  Sums are fp32. */
typedef struct {
    const void* y_dev; /* [n per_row][width] of `type` */
    int64_t y_ld;
    int32_t type;
    int32_t width;     /* 1..2^20 */
    int64_t n;
    int32_t per_row, networks;
    const int32_t* ids_dev; /* [n][per_row] */
    const float* w_dev;     /* [n][per_row] */
} pnn_combine;

/* out_dev [n][width] of out_type. */
pnn_status pnn_combine_rows(const pnn_combine* args, void* out_dev, int64_t out_ld, int32_t out_type, void* hip_stream);

/* From g_dev [n][width] of g_type, the gradient of out: dy[p] = w[p] g[r] (of `type`) and dw[p] =
 * sum g[r] y[p] (fp32), both 0 for a dropped pair.  dy_dev may be y_dev (with the same distance between rows). */
pnn_status pnn_combine_grad(const pnn_combine* args, const void* g_dev, int64_t g_ld, int32_t g_type, void* dy_dev, int64_t dy_ld,
                            float* dw_dev, void* hip_stream);

/* ---------------------------------------------------------------------------------------------
 * A step of AdamW over many tensors, beside the SGD of the training calls: for networks that a program
 * trains with the gradients above.  With step number t, which the call counts on the device,
 *   m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2
 *   p <- p (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32.  Parameters are fp32, with a bf16 copy (rounded to nearest even) where the products read one.
 * Moments are fp32 (bits = 32) or 8-bit codes (bits = 8), a byte a value and a scale for each 256 values of
 * a tensor: the largest |m| or v among them.  m's byte is a sign (the high bit) and a code c of 127, v's a code of 255:
 * 0 stands for 0, another for scale * 2^((c - 127) / 8) or 2^((c - 255) / 8).  A step takes the moments
 * before they are rounded.  Rounding goes up or down at random in proportion (v's lowest code counts for
 * all below it), by bits that are a function of seed, t, the tensor's place in the call, and the value's place: the
 * same call gives the same bits.  A moment that is infinite or NaN makes its block's scale NaN.  States begin as zeros. */
typedef struct {
    float* p_dev;                     /* [n] */
    const void* g_dev;                /* [n] of g_type */
    void *m_dev, *v_dev;              /* [n] fp32, or bytes */
    float *m_scale_dev, *v_scale_dev; /* [ceil(n / 256)] (bits = 8) */
    uint16_t* copy_dev;               /* [n] bf16, nullable */
    int64_t n;                        /* 0..2^40 */
} pnn_adamw_tensor;

/* A plan of the tensors (host array, read during the call; values are contiguous and aligned to their types): where a step
 * finds them, as long as they stay where they are.  Nothing that a step writes overlaps; a gradient may be its own tensor's p, m, v
 * or copy, value by value, and overlaps nothing else of these.  All have `bits` and g_type.  plan_dev is 16-byte aligned;
 * a program lays it out once. */
pnn_status pnn_adamw_bytes(const pnn_adamw_tensor* tensors, int32_t count, int64_t* bytes, int64_t* chunks);
pnn_status pnn_adamw_plan(const pnn_adamw_tensor* tensors, int32_t count, int32_t bits, int32_t g_type, void* plan_dev,
                          int64_t plan_bytes, void* hip_stream);

typedef struct {
    void* plan_dev;       /* written by pnn_adamw_plan; a step counts its workgroups there */
    int64_t chunks;       /* as pnn_adamw_bytes gives them */
    int32_t bits;         /* 32 or 8, and the gradients' type, as the plan was laid out: with others a step does */
    int32_t g_type;       /* nothing, and is not counted */
    double lr;            /* 0..1e6 */
    double beta1, beta2;  /* in [0, 1) */
    double eps;           /* 1e-30..1 */
    double weight_decay;  /* 0..1e6 */
    const float* lr_dev;  /* (nullable) [1], read by the step instead of lr: a recorded step's rate may change */
    uint32_t seed;
    int32_t* steps_dev;   /* [2]: the steps done so far, and 0 (the library's own during a call) */
} pnn_adamw;

/* One step of all tensors of a plan, in one launch.  Calls that share tensors, a plan or steps_dev are ordered by the caller.  May
 * be recorded into a graph. */
pnn_status pnn_adamw_step(const pnn_adamw* args, void* hip_stream);

/* What the 8-bit states of n values stand for, in fp32. */
pnn_status pnn_adamw_values(const uint8_t* m_dev, const uint8_t* v_dev, const float* m_scale_dev, const float* v_scale_dev, int64_t n,
                            float* m_out_dev, float* v_out_dev, void* hip_stream);

/* ---------------------------------------------------------------------------------------------
 * Distillation: a network learns another's answers (a way to combine CNs beside averaging them).
 * Row r has `classes` logits z, a teacher's `top` entries (class idx, logit t) and a label y.
 *   p = softmax(t / T) over the row's entries, q = softmax(z / T), s = softmax(z):
 *   loss = (1 - alpha) T^2 sum_j p_j (log p_j - log q_{idx_j}) - alpha log s_y
 *   dz_v = g [ (1 - alpha) T (q_v - sum_{j: idx_j = v} p_j) + alpha (s_v - [v = y]) ]
 * (with alpha = 1 the cross-entropy cost of eq. (6) and the output error of eq. (10)).  An entry
 * whose class lies outside [0, classes) is padding; one class may stand twice; a teacher logit of
 * -inf has no weight.  A label outside [0, classes) is none.  A row without entries and without a
 * label, and one whose logits are all -inf, has loss 0 and gradient 0; its logits may hold
 * anything in the first case.  z, t and dz are of `type`; sums and statistics are fp32, and the
 * maximum is subtracted first, so logits near the type's limits do not overflow (a class further below
 * the maximum than fp32's range counts as one of -inf).  Logarithms and quotients are rounded before T
 * scales them, so a loss is off by about 2^-22 (1 - alpha) T^2 and dz_v by 2^-22 g (1 - alpha) T q_v, which
 * at temperatures of thousands is as much as is left of them.  The order of the sums depends on the sizes
 * alone.  No handle, as for the grouped products above. */
typedef struct {
    const void* z_dev;      /* [n][classes] */
    int64_t z_ld;
    int32_t type;
    int32_t classes;        /* 1..2^30 */
    int64_t n;
    const int32_t* idx_dev; /* [n][top] */
    const void* t_dev;      /* [n][top] */
    int32_t top;            /* 0..1024 */
    const int32_t* y_dev;   /* [n]; read if alpha > 0 */
    float temperature;      /* T, 1e-6..1e6 */
    float alpha;            /* 0..1 */
} pnn_distill;

/* Size of the statistics that pnn_distill_loss leaves for pnn_distill_grad. */
pnn_status pnn_distill_bytes(int64_t n, int32_t classes, int64_t* bytes);

/* loss_dev [n] fp32, and the statistics (16-byte aligned). */
pnn_status pnn_distill_loss(const pnn_distill* args, float* loss_dev, void* stats_dev, int64_t stats_bytes, void* hip_stream);

/* dz_dev [n][classes] from the same arguments and their statistics; g_dev [n] is the gradient of
 * each row's loss (NULL: 1).  A row whose g is 0 gets 0, whatever its logits.  dz_dev may be z_dev
 * (with the same distance between rows). */
pnn_status pnn_distill_grad(const pnn_distill* args, const float* g_dev, const void* stats_dev, int64_t stats_bytes, void* dz_dev,
                            int64_t dz_ld, void* hip_stream);

/* ---------------------------------------------------------------------------------------------
 * A handle's child networks on rows that name them (at most 1,024 CNs: PNN_EINVAL otherwise).  Both
 * calls keep their grouping, activations and errors in one workspace of the handle that grows with the
 * pairs of a call, so calls of one handle on different streams have to be ordered by the caller; they
 * may be recorded into a graph as the other calls are (see the top), but not while a merge's broadcast
 * is still to be made (the fused last-layer plan: PNN_EHIP, nothing recorded).  x_dev
 * [rows][sizes[0]] fp32, ids_dev [rows][per_row] as in pnn_group_rows.  Products, activations and
 * roundings are those of pnn_infer and pnn_train_epoch up to the order of the fp32 sums. */

/* Answers of several networks combined (a combination of outputs where pnn_merge combines weights):
 * out_dev[r] (nullable) [rows][sizes[L]] = sum_j weights_dev[r per_row + j] x^L of pair j over the
 * row's pairs that are not dropped (weights NULL: their mean); pred_dev[r] its argmax (lowest index
 * on ties).  A row whose pairs are all dropped gets 0 and the class -1. */
pnn_status pnn_infer_routed(pnn_net* net, const float* x_dev, int64_t rows, const int32_t* ids_dev, int32_t per_row,
                            const float* weights_dev, int32_t* pred_dev, float* out_dev, void* hip_stream);

/* One mini-batch step of every CN on the pairs that name it (the configured batch size plays no
 * part), towards a teacher's top logits and labels: the loss of pnn_distill_loss at the pair's
 * output sums z^L, gradients averaged over the CN's pairs, W <- W - eta / pairs * gradient.  Row r's
 * pairs share its entries idx_dev, t_dev [rows][top] (fp32) and its label y_dev [rows] (read if
 * alpha > 0).  alpha = 1 is the step of pnn_train_epoch.  Needs a softmax output layer (PNN_EINVAL).
 * A CN without pairs keeps its parameters; the merged network keeps its own.  loss_dev (nullable)
 * [rows per_row] receives the pairs' losses before the step, 0 for dropped ones. */
pnn_status pnn_train_routed(pnn_net* net, const float* x_dev, int64_t rows, const int32_t* ids_dev, int32_t per_row,
                            const int32_t* idx_dev, const float* t_dev, int32_t top, const int32_t* y_dev, float temperature,
                            float alpha, float* loss_dev, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* PNN_H */
