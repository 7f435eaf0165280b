/*
 * qlayer.h -- C ABI of the batched quantum-layer library (HIP, gfx950).
 *
 * The library simulates a batch of parameterised quantum circuits on one
 * GPU and returns what the paper's quantum node hands to the rest of a hybrid
 * network (Sec. "Quantum Node"): the measured outputs in the forward pass and,
 * for back-propagation (Sec. "Optimization", hybrid optimisation), the
 * gradient of the loss with respect to the circuit parameters. The quantum
 * node's backward returns the gradient multiplied by the upstream gradient
 * (appendix, hybrid quantum-classical network, class Hybrid), i.e. a
 * vector-Jacobian product. The angles of the rotation gates are bound either
 * to input features (angle encoding, Sec. "Quantum Data") or to trainable
 * weights shared by every sample of the batch.
 *
 * Conventions
 *   - qubit q is bit q of the amplitude index; the initial state is |0...0>;
 *   - H = [[1,1],[1,-1]]/sqrt(2); RX(t), RY(t), RZ(t) = exp(-i t P / 2) for
 *     P = X, Y, Z; CNOT(q0 = control, q1 = target); CZ(q0, q1);
 *   - expz[b][i] is the exact expectation <Z_i> of sample b (the limit of
 *     infinitely many measurement shots), no renormalisation;
 *   - grad_inputs[b][f]  = sum_i grad_out[b][i] d expz[b][i] / d inputs[b][f]
 *     grad_weights[p]    = sum_b sum_i grad_out[b][i] d expz[b][i] / d weights[p]
 *     (every occurrence of an input or weight in the gate list adds up);
 *   - gradients are computed by adjoint differentiation (one reverse sweep
 *     that un-applies the gates and accumulates Im<lambda|P|psi> per rotation).
 *
 * Precision: QL_C64 states are complex64 (fp32 real/imag), angles, grad_out
 * and all outputs are fp32; QL_C128 uses complex128 and fp64 throughout.
 * Every reduction runs in a fixed order, so results are bit-reproducible run
 * to run. For QL_C64, sums over one wavefront and over the tiles of one
 * workgroup are fp32; sums across wavefronts, workgroups and the batch are
 * fp64.
 *
 * Memory: all array arguments of ql_forward / ql_forward_backward are DEVICE
 * pointers on the current HIP device, row-major and contiguous, owned by the
 * caller. The caller also provides the device workspace (size from
 * ql_workspace_bytes). The library writes only the workspace and the outputs.
 * It allocates device memory in one place: the first call of a dtype on a
 * handle and device queues a device copy of the handle's plan tables (some KiB),
 * which later calls read and ql_circuit_destroy frees.
 * Until that copy has arrived, and where no device memory may be
 * allocated (a stream in capture, ql_forward_backward_static), an allocation
 * fails, or the stream belongs to another device than the current one, the call
 * copies the tables to the workspace instead. A graph captured from calls on a
 * handle reads the handle's tables when it is replayed: keep the handle until
 * the last replay has ended. Outputs are
 * overwritten (not accumulated). Buffers must not alias each other or the
 * workspace.
 *
 * Errors: every function returns QL_OK (0) or a negative QL_E* code and sets a
 * thread-local message readable with ql_last_error(). All argument checks
 * happen before anything is launched. Calls are asynchronous on the given
 * stream; results are valid once the stream has been synchronised. A circuit
 * handle is immutable after creation and may be used from several threads and
 * streams at once, each with its own workspace.
 */
#ifndef QLAYER_H
#define QLAYER_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Gate kinds.
 *
 * QL_CRX/QL_CRY/QL_CRZ (q0 = control, q1 = target): the rotation of the
 * target on the amplitudes whose control bit is 1, |0><0| (x) I + |1><1| (x)
 * R(t) -- the controlled rotations of the paper's quantum autoencoder
 * (appendix "Quantum Autoencoder"). Their gradient is exact (generator
 * |1><1| (x) P).
 *
 * QL_PAULI (q0, q1 = -1, src = QL_SRC_INPUT): one quantum trajectory of a
 * Pauli channel, the noise model of the paper's noise-inclusive simulator
 * (Sec. "Unification of Classical and Quantum Machine"). With the channel's
 * probabilities (p_x, p_y, p_z) (ql_circuit_desc.pauli_p) and the sample's
 * uniform u = inputs[b][index] in [0, 1), it applies X if u < p_x, else Y if
 * u < p_x + p_y, else Z if u < p_x + p_y + p_z, else nothing (fp64 sums in that
 * order). The mean of <Z> over samples with independent uniforms estimates
 * the noisy expectation; the uniform gets no gradient. */
enum { QL_H = 0, QL_RX = 1, QL_RY = 2, QL_RZ = 3, QL_CNOT = 4, QL_CZ = 5,
       QL_CRX = 6, QL_CRY = 7, QL_CRZ = 8, QL_PAULI = 9 };

/* Where a rotation angle comes from: H/CNOT/CZ use QL_SRC_NONE; RX/RY/RZ and
 * the controlled rotations use QL_SRC_INPUT (feature `index` of each sample)
 * or QL_SRC_WEIGHT (trainable weight `index`). */
enum { QL_SRC_NONE = 0, QL_SRC_INPUT = 1, QL_SRC_WEIGHT = 2 };

/* One gate. One-qubit gates use q0 and set q1 = -1. */
typedef struct {
    int32_t kind, q0, q1, src, index;
} ql_gate;

/* Initial-state embeddings (Sec. "Quantum Data": encoding classical data into
 * the basis state or into the amplitude vector; angle encoding is rotation
 * gates bound to inputs).
 *   QL_EMBED_NONE       |0...0>.
 *   QL_EMBED_BASIS      qubit q is 1 where inputs[b][first + q] >= 0.5 (a
 *                       direct-product basis state); no gradient.
 *   QL_EMBED_AMPLITUDE  psi_0 = x / |x| for the 2^n real features
 *                       x = inputs[b][first .. first + 2^n - 1] (n <= 30; a
 *                       zero vector gives the zero state: <Z> = 0, no
 *                       gradient). grad_inputs of those features is the VJP
 *                       through the normalisation,
 *                       (2 / |x|) (Re lambda_0 - psi_0 Re<psi_0|lambda_0>),
 *                       with lambda_0 the adjoint state after the sweep. */
enum { QL_EMBED_NONE = 0, QL_EMBED_BASIS = 1, QL_EMBED_AMPLITUDE = 2 };

/* Circuit extras for ql_circuit_create_desc. pauli_p[c][3] = (p_x, p_y, p_z)
 * of the c-th QL_PAULI gate in gate order (each >= 0, sum <= 1); read during
 * the call only. NULL when the circuit has no Pauli channels. */
typedef struct {
    int32_t embedding;      /* QL_EMBED_* */
    int32_t embed_first;    /* first input feature the embedding reads */
    const double* pauli_p;
} ql_circuit_desc;

typedef enum { QL_C64 = 0, QL_C128 = 1 } ql_dtype;

/* Workspace modes. QL_MODE_FWD_BWD_KEEP is ql_forward_backward with the
 * state after every tile pass but the last kept in the workspace: the
 * backward pass over tile pass p+1 then leaves its un-computed state unstored
 * and the one over pass p loads the kept state after pass p instead (one
 * state write fewer per backward pass: 5m - 5 instead of 6m - 6 state
 * transfers for m tile passes), at the cost of m - 2 more states of
 * workspace (m - 1 with an embedding, whose initial state keeps its
 * buffer). ql_forward_backward takes this path whenever its workspace holds
 * ql_workspace_bytes(..., QL_MODE_FWD_BWD_KEEP) bytes; results agree with the
 * other path up to rounding (the backward reads the forward's states rather
 * than re-derived ones). With one tile pass (or the whole-state kernel) there
 * is nothing to keep; with two the kept state takes the place of the psi
 * buffer, the two sizes are equal and the states are always kept. */
enum { QL_MODE_FWD = 0, QL_MODE_FWD_BWD = 1, QL_MODE_FWD_BWD_KEEP = 2 };

enum {
    QL_OK = 0,
    QL_EINVAL = -1,       /* invalid argument (gate, index, pointer, size) */
    QL_ENOMEM = -2,       /* workspace too small, size overflow, host allocation failed */
    QL_EUNSUPPORTED = -3, /* too many qubits for this dtype or option out of range */
    QL_EHIP = -4          /* HIP runtime error (message from hipGetErrorString) */
};

/* Largest qubit count per dtype. */
#define QL_MAX_QUBITS_C64 32
#define QL_MAX_QUBITS_C128 31

/* Optional planning knobs; zero means "library default". They change how the
 * work is split into kernel passes, never the results beyond fp rounding. */
typedef struct {
    int32_t log_regs;           /* amplitudes per thread = 2^log_regs (2..5) */
    int32_t log_threads;        /* threads per workgroup = 2^log_threads (6..9) */
    int32_t low_qubits;         /* qubits 0..low_qubits-1 are in every tile (1..8) */
    int32_t max_gates_per_pass; /* cap on gates per tile pass (>= 1) */
    int32_t force_tiled;        /* kernel choice: 0 library default (the run kernel for
                                   n <= 12 where it fits and pays, see
                                   ql_call_kernel; else register tiles for n >= 8, a
                                   whole-state kernel below), 1 register tiles for
                                   n >= 8, -1 a whole-state kernel whenever it fits
                                   (n <= 12 for QL_C64, n <= 11 for QL_C128). The
                                   whole-state kernels hold a sample in one
                                   wavefront's registers for n <= 8 (in LDS for
                                   forward-only launches of 2048 or more circuits)
                                   and in LDS above */
    int32_t wg_per_sample;      /* workgroups per sample in a tile pass */
    int32_t rz_groups;          /* 0: RZs on the register bits of one tile layout that
                                   commute into one place (at least three, on distinct
                                   bits) run as one per-register phase op, and an RZ
                                   that commutes back to an RY on its bit runs in one
                                   op with it; -1: every RZ runs on its own */
    int32_t pass_search;        /* how the tiles of the passes are chosen. 1: one pass
                                   at a time, the candidate whose pass plus a greedy
                                   completion of the rest is cheapest under a
                                   memory/arithmetic cost model (no nearly empty
                                   passes at the end of long CNOT chains); -1: one
                                   pass at a time, the candidate that runs the most
                                   gates; 0 (default): a beam search over whole pass
                                   sequences, taken when it needs fewer passes than
                                   1, else 1 */
    int32_t product_prefix;     /* the one-qubit gates a qubit meets before any
                                   two-qubit gate or Pauli channel touches it (the
                                   product-state prefix of the circuit) need not
                                   run as tile ops: the first pass can start from
                                   the product state they make (per-sample
                                   factors, fp64), and their gradients come from
                                   each qubit's environment in lambda at the end of
                                   the backward sweep (tile plans without an
                                   embedding). 0 (default): so when the other gates
                                   then plan into fewer passes, or as many with no
                                   more layout changes; 1: always; -1: never */
    int32_t cz_groups;          /* 0: two or more CZs of one tile layout that commute
                                   into one place (each with at least one operand
                                   outside the registers, or on two register bits)
                                   run as one sign op; -1: every CZ runs on its own */
} ql_options;

typedef struct ql_circuit ql_circuit; /* opaque */

/* Validate the gate list and build the pass plans for both dtypes.
 * n_qubits in [1, 32]; gates[n_gates] as above; n_inputs features per sample
 * and n_weights trainable weights index the angle sources. The gate list is
 * copied. Returns QL_EINVAL for a bad qubit, q0 == q1, a wrong source for the
 * kind, an index out of range or a NULL pointer. */
int ql_circuit_create(int32_t n_qubits, const ql_gate* gates, int32_t n_gates,
                      int32_t n_inputs, int32_t n_weights, ql_circuit** out);

/* Same with planning options (NULL = defaults). */
int ql_circuit_create_ex(int32_t n_qubits, const ql_gate* gates, int32_t n_gates,
                         int32_t n_inputs, int32_t n_weights, const ql_options* opts,
                         ql_circuit** out);

/* Same with an initial-state embedding and Pauli-channel probabilities (desc
 * NULL = no embedding, no channels) and planning options (NULL = defaults).
 * Returns QL_EINVAL also for an embedding whose features do not fit in
 * n_inputs, amplitude embedding above 30 qubits, a QL_PAULI gate without
 * probabilities, or probabilities < 0 or summing above 1. Every entry point
 * honours the embedding and the channels. */
int ql_circuit_create_desc(int32_t n_qubits, const ql_gate* gates, int32_t n_gates,
                           int32_t n_inputs, int32_t n_weights, const ql_circuit_desc* desc,
                           const ql_options* opts, ql_circuit** out);

/* Free a handle (NULL is a no-op). Freeing its plan tables waits for the queued
 * work of the devices it ran on. The handle must not be used afterwards. */
void ql_circuit_destroy(ql_circuit* c);

/* Bytes of device workspace a call with this dtype, batch and mode
 * (QL_MODE_*) needs. */
int ql_workspace_bytes(const ql_circuit* c, ql_dtype dtype, int64_t batch, int mode,
                       size_t* out);

/* Forward: inputs[batch][n_inputs], weights[n_weights] -> expz[batch][n_qubits].
 * inputs may be NULL when n_inputs == 0, weights when n_weights == 0. */
int ql_forward(const ql_circuit* c, ql_dtype dtype, int64_t batch,
               const void* inputs, const void* weights, void* expz,
               void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Forward + adjoint VJP. grad_out[batch][n_qubits] is the upstream gradient;
 * grad_inputs[batch][n_inputs] and grad_weights[n_weights] may each be NULL
 * (not computed). expz is written as in ql_forward. */
int ql_forward_backward(const ql_circuit* c, ql_dtype dtype, int64_t batch,
                        const void* inputs, const void* weights, const void* grad_out,
                        void* expz, void* grad_inputs, void* grad_weights,
                        void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Allocation-free forward + backward, for callers that cannot allocate
 * device memory or pass a workspace (code under HIP graph capture, tight
 * serving loops, harnesses that forbid allocation).
 *
 * Same arguments, results and errors as ql_forward_backward without the
 * workspace: the call runs in a static device buffer of
 * QL_STATIC_SCRATCH_BYTES that the library holds on every GPU it runs on
 * until the process ends, and returns QL_ENOMEM (before launching anything)
 * when the circuit, dtype and batch need more than that (they never do when
 * ql_workspace_bytes(..., QL_MODE_FWD_BWD) is no more; a tile plan may fit with
 * somewhat more, in a layout of less workspace). It calls no device or
 * host allocator: the plan tables are copied from the handle's own host copy.
 * The caller still provides inputs and outputs. All calls on one GPU share
 * that GPU's buffer: calls that overlap in time on one GPU (other streams,
 * other threads) race and give wrong results; serialise them. Nothing in the
 * buffer needs to start at zero, so its contents from an earlier call do not
 * matter. */
#define QL_STATIC_SCRATCH_BYTES (64u << 20)
int ql_forward_backward_static(const ql_circuit* c, ql_dtype dtype, int64_t batch,
                               const void* inputs, const void* weights, const void* grad_out,
                               void* expz, void* grad_inputs, void* grad_weights,
                               hipStream_t stream);
/* ---- parameter-shift gradients -------------------------------------------
 *
 * The same VJP as ql_forward_backward, computed with the two-term
 * parameter-shift rule instead of the adjoint sweep. The paper's hybrid example
 * (appendix, class Hybrid) differentiates its quantum node this way, by
 * re-running the circuit with the angle shifted by +pi/2 and -pi/2; for
 * exp(-i t P / 2) gates d<Z_i>/dt = (<Z_i>(t + pi/2) - <Z_i>(t - pi/2)) / 2 is
 * exact (the paper's own expression omits the 1/2). Every rotation occurrence
 * s of every sample b gives two shifted circuits; together with the unshifted
 * one these are B * (2S + 1) circuits for S rotation gates, run as extra
 * samples of batched forward passes in chunks of at most max_chunk circuits
 * (0 = all at once). Arguments, outputs, layout and errors are those of
 * ql_forward_backward; grad_out is required. The workspace must hold
 * ql_param_shift_workspace_bytes(c, dtype, batch, max_chunk) bytes; it grows
 * with the chunk (one state per circuit of a chunk) and with B * (2S + 1)
 * fp64 values. Results are deterministic.
 *
 * A controlled rotation CR(t) equals R(t/2) E R(-t/2) E (E = CNOT for CRY and
 * CRZ, CZ for CRX); its two half-angle rotations are shifted separately and
 * their differences combined with factors +-1/2, which is exact (it equals
 * the four-term rule for the controlled generator). Pauli channels are not
 * shifted. With QL_EMBED_AMPLITUDE, grad_inputs must be NULL
 * (QL_EUNSUPPORTED otherwise): the shift rule gives no gradient for
 * amplitudes. */
int ql_param_shift_workspace_bytes(const ql_circuit* c, ql_dtype dtype, int64_t batch,
                                   int64_t max_chunk, size_t* out);
int ql_param_shift(const ql_circuit* c, ql_dtype dtype, int64_t batch, const void* inputs,
                   const void* weights, const void* grad_out, void* expz, void* grad_inputs,
                   void* grad_weights, int64_t max_chunk, void* workspace,
                   size_t workspace_bytes, hipStream_t stream);

/* ---- final states and shot sampling --------------------------------------
 *
 * The paper's quantum node measures its circuit with a finite number of shots
 * (Sec. "Quantum Node"; the appendix examples measure 100 shots and turn the
 * counts into probabilities). These calls expose that measurement: ql_state
 * writes the final state of every sample, and ql_sample draws shots from
 * states with caller-supplied uniforms.
 *
 * ql_state: same inputs as ql_forward; psi[batch][2^n_qubits] receives the
 * final state (interleaved complex: float2 for QL_C64, double2 for QL_C128),
 * a caller-owned device buffer that also serves as the working state (the
 * workspace then holds no state). Workspace from ql_state_workspace_bytes. */
int ql_state_workspace_bytes(const ql_circuit* c, ql_dtype dtype, int64_t batch, size_t* out);
int ql_state(const ql_circuit* c, ql_dtype dtype, int64_t batch, const void* inputs,
             const void* weights, void* psi, void* workspace, size_t workspace_bytes,
             hipStream_t stream);

/* ql_sample: psi[batch][2^n_qubits] (device, the layout of ql_state) and
 * uniforms[batch][shots] (device, fp64 in [0, 1)); samples[batch][shots]
 * (device, int64) receives, for shot s of sample b, the smallest basis index j
 * whose running sum of |psi_i|^2 (i <= j, in index order) exceeds
 * uniforms[b][s] times the state's total |psi|^2 -- the inverse-CDF draw, so
 * the index's bits are the measured qubits (qubit q = bit q) and no
 * zero-probability index is returned. The sums run in fp64 in a fixed
 * (blocked) order; when a uniform falls within rounding of a CDF boundary the
 * neighbouring index may be returned. zhat[batch][n_qubits] (device, fp32 for
 * QL_C64, fp64 for QL_C128; may be NULL) receives the shot estimate of <Z_q>:
 * (shots with bit q = 0 minus shots with bit q = 1) / shots. The states need
 * not be normalised. shots = 0 writes nothing. Workspace:
 * ql_sample_workspace_bytes(n_qubits, batch) bytes (per block of up to 4096
 * amplitudes, the prefix of block totals and the block's 64 chunk sums:
 * 65 fp64). n_qubits in [1, 32] (QL_C128: [1, 31]). */
int ql_sample_workspace_bytes(int32_t n_qubits, int64_t batch, size_t* out);
int ql_sample(ql_dtype dtype, int32_t n_qubits, int64_t batch, const void* psi, int64_t shots,
              const double* uniforms, int64_t* samples, void* zhat, void* workspace,
              size_t workspace_bytes, hipStream_t stream);

/* ---- operators around a quantum layer -------------------------------------
 *
 * What a hybrid network needs on either side of its quantum layer: a norm that
 * brings features to the range of angles, with its gradients, and the
 * optimiser's step of matrix-shaped weights. They need no
 * circuit, allocate nothing, keep nothing between calls, run on the given
 * stream and can be captured in a graph. Pointers are device addresses that are
 * multiples of the element's size; outputs and the workspace overlap nothing. */

/* Element types. Statistics and sums are fp64 for QL_F64 and fp32 otherwise
 * (fp64 where sums of workgroups are joined); outputs are rounded once. */
typedef enum { QL_F32 = 0, QL_F64 = 1, QL_BF16 = 2, QL_F16 = 3 } ql_type;

/* Layer norm of rows of features:
 *   y = (x - mean) * rstd * weight + bias,  mean = sum x / features,
 *   rstd = 1 / sqrt(sum (x - mean)^2 / features + eps).
 * x holds rows that start x_stride elements apart (>= 0: rows may be columns of
 * a wider array, or one row repeated); y[rows][features] is contiguous.
 * weight[features] and bias[features] (weight_type: type, or QL_F32 beside
 * QL_BF16 and QL_F16 rows) may each be NULL (1 and 0). mean[rows] and
 * rstd[rows] (QL_F64 for QL_F64, else QL_F32) are what the backward call needs
 * and may each be NULL. A row that holds an infinity or NaN, or with eps = 0 no
 * variance, gives NaN in that row alone. features in [1, 2^30]; rows = 0 does
 * nothing.
 *
 * The backward call: with h = (x - mean) * rstd,
 *   grad_x      = rstd * (g w - mean(g w) - h * mean(g w h)),
 *   grad_weight = sum over rows of g h,   grad_bias = sum over rows of g,
 * each of which may be NULL (not computed); grad_y's rows start grad_stride
 * elements apart, grad_x[rows][features] is contiguous. Sums over rows run in a
 * fixed order.
 *
 * ql_layer_norm_workspace_bytes gives the device workspace of a forward
 * (backward = 0) or backward call; where it is 0, as for forward calls of
 * ordinary rows, the workspace may be NULL. */
int ql_layer_norm_forward(ql_type type, ql_type weight_type, int64_t rows, int64_t features,
                          const void* x, int64_t x_stride, const void* weight, const void* bias,
                          double eps, void* y, void* mean, void* rstd, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);
int ql_layer_norm_workspace_bytes(ql_type type, int64_t rows, int64_t features, int backward,
                                  size_t* out);
int ql_layer_norm_backward(ql_type type, ql_type weight_type, int64_t rows, int64_t features,
                           const void* grad_y, int64_t grad_stride, const void* x, int64_t x_stride,
                           const void* mean, const void* rstd, const void* weight, void* grad_x,
                           void* grad_weight, void* grad_bias, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* Orthogonalised updates of matrix-shaped weights (the layers around a quantum
 * layer, or its own angles as [layers][angles of a layer]).
 *
 * O = orthogonalised U: X = U / (|U|_F + eps), turned so that it has no more
 * rows than columns, then `steps` times
 *   A = X X^T,   X = a X + (b A + c A^2) X,
 * which takes every singular value s of X through a s + b s^3 + c s^5 towards 1
 * and leaves the singular vectors. A matrix of zeros gives zeros (NaN with eps
 * = 0); one that holds an infinity or NaN gives NaN throughout.
 *
 * ql_orthogonalize: U = grad, out = O.
 * ql_muon_step: momentum = mu * momentum + grad, U = grad + mu * momentum (with
 * nesterov; else U = momentum), out = (1 - lr * weight_decay) * out
 * - lr * sqrt(max(1, rows / cols)) * O, all in place.
 *
 * An entry is `batch` matrices of rows x cols; each array has its strides in
 * elements between matrices, rows and columns (any order; >= 0, and out and
 * momentum must not overlap themselves). grad and out are of `type`; momentum
 * (unused by ql_orthogonalize) is QL_F64 for QL_F64 and QL_F32 otherwise. out may
 * be grad's array in ql_orthogonalize where the strides are equal. All entries of
 * a call run together: give a network's matrices in one call.
 *
 * Precision: QL_F64 in fp64 (updates whose squares leave its range are not
 * scaled). Other products are fp16 ones that keep 22 bits of every factor (in two
 * parts); sums are fp32, norms fp64. A matrix's last bits can depend on what else
 * the call holds (the tiles follow from all of it), and nothing else: the same
 * call gives the same bits.
 *
 * options NULL: the defaults in braces. rows, cols in [1, 65536], steps in
 * [1, 64]; coefficients that let a singular value in [0, 1] grow past 64 before
 * the last step are refused, and so are 2^23 or more 64x64 blocks of matrices of
 * which one is too large for a workgroup's LDS. The entries are read during the
 * call only. */
typedef struct {
    int64_t rows, cols, batch;
    const void* grad;
    int64_t grad_stride[3];
    void* momentum;
    int64_t momentum_stride[3];
    void* out;
    int64_t out_stride[3];
} ql_matrix;

typedef struct {
    double a, b, c;   /* {3.4445, -4.7750, 2.0315} */
    double eps;       /* {1e-7} */
    int32_t steps;    /* {5} */
} ql_ortho_options;

typedef struct {
    double lr, momentum, weight_decay; /* {0.02, 0.95, 0} */
    int32_t nesterov;                  /* {1} */
} ql_muon_options;

int ql_orthogonalize_workspace_bytes(ql_type type, const ql_matrix* matrices, int32_t count,
                                     size_t* out);
int ql_orthogonalize(ql_type type, const ql_matrix* matrices, int32_t count,
                     const ql_ortho_options* options, void* workspace, size_t workspace_bytes,
                     hipStream_t stream);
/* Same workspace as ql_orthogonalize. */
int ql_muon_step(ql_type type, const ql_matrix* matrices, int32_t count,
                 const ql_muon_options* muon, const ql_ortho_options* options, void* workspace,
                 size_t workspace_bytes, hipStream_t stream);

/* ---- operators of a network that reads sequences ---------------------------
 *
 * What stands in front of a quantum layer where features come from sequences of
 * tokens. As the operators above: no circuit, no allocation, nothing kept, the
 * given stream, capture in a graph, pointers that are multiples of the element's
 * size, outputs and the workspace overlap nothing. Sums are fp64 for QL_F64 and fp32
 * otherwise (fp64 where sums of workgroups are joined), in a fixed order. */

/* Root-mean-square norm of rows of features, with the residual's addition:
 *   s = x + residual (rounded to its type),  rstd = 1 / sqrt(sum s^2 / features + eps),
 *   y = s * rstd * weight.
 * Rows of x and residual start x_stride and residual_stride elements apart (>= 0);
 * summed[rows][features] = s and y[rows][features] are contiguous. residual may
 * be NULL (s = x, and summed is not written), weight too (1); its type is the
 * rows', or QL_F32 beside 16-bit rows. rstd[rows] (QL_F64 for QL_F64, else
 * QL_F32) is what the backward call needs and may be NULL. A row that holds NaN
 * gives NaN in that row alone; one whose sum of squares is infinite has rstd 0, as
 * the formula says (zeros, and NaN for an infinity itself). features in [1, 2^30];
 * rows = 0 does nothing.
 *
 * scale not NULL: y is bytes in e4m3 (OCP FP8, largest value 448) instead, and
 * scale[rows] (QL_F32) = max |s * rstd * weight| / 448 is what they are multiples of; a
 * row of zeros has scale 0, and where the row holds an infinity or NaN the scale is
 * NaN. The bytes are s * weight * 448 / max |s * weight| to nearest, halves to even: as
 * defined for QL_BF16 rows and weights, otherwise of a value that may be off by 2^-20 of
 * itself. Not for QL_F64 (QL_EUNSUPPORTED).
 *
 * The backward call: with h = s * rstd,
 *   grad_x      = rstd * (g w - h * mean(g w h)) + grad_summed (NULL: 0),
 *   grad_weight = sum over rows of g h,
 * each of which may be NULL (not computed). grad_x is the residual's gradient too.
 * The rows of s, grad_y and grad_summed start their strides apart.
 *
 * ql_rms_norm_workspace_bytes gives the device workspace of a forward (backward
 * = 0) or backward call; where it is 0 the workspace may be NULL. */
int ql_rms_norm_forward(ql_type type, ql_type weight_type, int64_t rows, int64_t features,
                        const void* x, int64_t x_stride, const void* residual,
                        int64_t residual_stride, const void* weight, double eps, void* summed,
                        void* y, void* rstd, float* scale, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);
int ql_rms_norm_workspace_bytes(ql_type type, int64_t rows, int64_t features, int backward,
                                size_t* out);
int ql_rms_norm_backward(ql_type type, ql_type weight_type, int64_t rows, int64_t features,
                         const void* grad_y, int64_t grad_stride, const void* grad_summed,
                         int64_t grad_summed_stride, const void* s, int64_t s_stride,
                         const void* rstd, const void* weight, void* grad_x, void* grad_weight,
                         void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Embedding: y_i = scale * W[t_i] for `count` tokens, W of rows x features whose rows
 * start weight_stride elements apart, y[count][features] contiguous. Tokens are int64
 * (tokens_64 not 0) or int32. With has_padding, tokens equal to `padding` (in the
 * table or not) give zeros. Other tokens outside [0, rows) give NaN.
 *
 * The backward call: grad_weight[v] = scale * (sum over i with t_i = v of grad_y_i),
 * [rows][features] contiguous, added in an order that the call's tokens fix: the same
 * bits every time (with other tokens beside it a row's sum may be rounded otherwise). Tokens
 * that are the padding or outside the table have no gradient, rows without tokens get zeros.
 *
 * count in [0, 2^31), rows in [1, 2^31), features in [1, 2^22], scale finite (as
 * QL_F32 where the rows are not QL_F64).
 * ql_embedding_workspace_bytes gives the backward call's device workspace. */
int ql_embedding_forward(ql_type type, int tokens_64, int64_t count, int64_t rows, int64_t features,
                         const void* tokens, const void* weight, int64_t weight_stride,
                         double scale, int has_padding, int64_t padding, void* y,
                         hipStream_t stream);
int ql_embedding_workspace_bytes(ql_type type, int64_t count, int64_t rows, int64_t features,
                                 size_t* out);
int ql_embedding_backward(ql_type type, int tokens_64, int64_t count, int64_t rows,
                          int64_t features, const void* tokens, const void* grad_y,
                          int64_t grad_stride, double scale, int has_padding, int64_t padding,
                          void* grad_weight, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/* Dropout: y_i = x_i / (1 - p) where word(i) >= p * 2^32 (rounded), 0 elsewhere
 * whatever x_i is. i is the element's place in row-major order, word(i) word i mod
 * 4 of Philox 4x32 with 10 rounds of the counter (i / 4, offset), low words first, under
 * the key seed: the mask depends on nothing else, and the gradient is the same call
 * on grad_y. p in [0, 1]; 1 gives zeros. key NULL, or the device address of seed and
 * offset, which are then read when the kernel runs (a graph's replays draw new masks
 * if the caller changes them) in place of the arguments. x's rows start x_stride
 * elements apart, y[rows][features] is contiguous. features in [1, 2^30]; rows = 0
 * does nothing. */
int ql_dropout(ql_type type, int64_t rows, int64_t features, const void* x, int64_t x_stride,
               double p, uint64_t seed, uint64_t offset, const uint64_t* key, void* y,
               hipStream_t stream);

/* Gated linear recurrence over the steps of sequences:
 *   a_t = 1 / (1 + exp(-gate_t)),  h_t = a_t h_{t-1} + (1 - a_t) x_t.
 * x and gate are [batch][steps][features] arrays whose sequences and steps start
 * x_batch and x_step (gate_batch, gate_step) elements apart (>= 0: the halves of one
 * projection, say); h is contiguous. States are QL_F64 for QL_F64 and QL_F32
 * otherwise: initial[batch][features] before the first step (NULL: 0), last[batch]
 * [features] after the last one (may be NULL), and for the backward call states[batch]
 * [ceil(steps / QL_SCAN_BLOCK)][features], the state before every QL_SCAN_BLOCK
 * steps (may be NULL). starts[batch][steps] (may be NULL) is not 0 where a sequence
 * begins: the state before that step is taken as 0, whatever it holds. A state that is not finite
 * makes its sequence's later ones infinite or NaN, and no others.
 *
 * The backward call: with G_t = grad_h_t + a_{t+1} G_{t+1} (behind the last step
 * grad_last, which may be NULL; nothing comes back past a start),
 *   grad_x = (1 - a) G,  grad_gate = G (h_{t-1} - x) a (1 - a),  grad_initial = a_0 G_0
 * (may be NULL). grad_x and grad_gate are contiguous.
 *
 * The step call is one step of each sequence: x and gate [batch] rows x_batch and
 * gate_batch elements apart, starts[batch], state[batch][features] in place,
 * h[batch][features].
 *
 * features in [1, 2^22], steps in [0, 2^30], batch * features in [0, 2^27]; batch = 0 does
 * nothing. ql_gated_scan_workspace_bytes gives the device workspace of a forward or
 * backward call; where it is 0 the workspace may be NULL. */
#define QL_SCAN_BLOCK 16
int ql_gated_scan_forward(ql_type type, int64_t batch, int64_t steps, int64_t features,
                          const void* x, int64_t x_batch, int64_t x_step, const void* gate,
                          int64_t gate_batch, int64_t gate_step, const uint8_t* starts,
                          const void* initial, void* h, void* last, void* states,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);
int ql_gated_scan_workspace_bytes(ql_type type, int64_t batch, int64_t steps, int64_t features,
                                  size_t* out);
int ql_gated_scan_backward(ql_type type, int64_t batch, int64_t steps, int64_t features,
                           const void* grad_h, int64_t grad_batch, int64_t grad_step,
                           const void* x, int64_t x_batch, int64_t x_step, const void* gate,
                           int64_t gate_batch, int64_t gate_step, const void* states,
                           const uint8_t* starts, const void* grad_last, void* grad_x,
                           void* grad_gate, void* grad_initial, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);
int ql_gated_scan_step(ql_type type, int64_t batch, int64_t features, const void* x,
                       int64_t x_batch, const void* gate, int64_t gate_batch,
                       const uint8_t* starts, void* state, void* h, hipStream_t stream);

/* Message of the last failing call on this thread ("" if none). */
const char* ql_last_error(void);

/* ---- introspection (host only, no GPU needed) ---------------------------- */

typedef struct {
    int32_t kernel;        /* plan of the handle: 0 = whole state on chip (one workgroup per sample), 1 =
                              tile passes. Calls of small circuits may take the run kernel
                              instead: ql_call_kernel tells */
    int32_t n_passes;      /* forward tile passes (1 for the whole-state kernel) */
    int32_t tile_qubits;   /* qubits per tile (log2 amplitudes per workgroup tile) */
    int32_t log_regs;      /* amplitudes per thread = 2^log_regs */
    int32_t log_threads;   /* threads per workgroup = 2^log_threads */
    int32_t low_qubits;    /* contiguous low qubits in every tile */
    int32_t n_transposes;  /* LDS layout changes summed over the forward passes */
    int32_t n_param_gates; /* rotation occurrences bound to inputs or weights (S of the
                              parameter-shift count; a controlled rotation counts 2) */
    int32_t n_lane_swaps;  /* in-register layout changes (register bit <-> lane bit) summed
                              over the forward passes */
    int32_t n_rz_groups;   /* RZ groups (several RZs run as one phase op), all passes */
    int32_t n_ryz_pairs;   /* RZs run together with their bit's RY in one op, all passes */
    int32_t n_prefix_gates; /* gates of the product-state prefix (the first pass's initial
                               state; see ql_options.product_prefix) */
    int32_t n_cz_groups;   /* CZ groups (several CZs run as one sign op), all passes */
} ql_plan_info;

int ql_plan_info_get(const ql_circuit* c, ql_dtype dtype, ql_plan_info* out);

/* Which kernel the state of a call runs in: QL_KERNEL_RUNS is the run kernel
 * (n <= 12: one workgroup per sample, the whole call in one launch, runs of
 * one-qubit gates as one matrix), the others the handle's plan
 * (ql_plan_info.kernel). mode: QL_MODE_*, or QL_CALL_STATE for ql_state;
 * ql_param_shift runs its chunks as QL_MODE_FWD of that many samples. The run
 * kernel takes circuits below 8 qubits unless force_tiled is -1, and of 8 to 12
 * qubits when every planning option is at its default (the options describe
 * tile plans), where its tables fit and the batch is not too large for it;
 * complex64 final states never. */
enum { QL_KERNEL_WHOLE = 0, QL_KERNEL_TILE = 1, QL_KERNEL_RUNS = 2 };
enum { QL_CALL_STATE = 3 };
int ql_call_kernel(const ql_circuit* c, ql_dtype dtype, int64_t batch, int mode, int32_t* out);

/* Forward schedule: pass_of_gate[n_gates] receives the pass that applies each
 * gate, order[n_gates] the gate indices in execution order (pass by pass).
 * Gates of the product-state prefix belong to pass 0 and come first, in gate
 * order. A controlled rotation or Pauli channel runs as several gates; it is
 * reported at the pass and position of the last one (a channel with all
 * probabilities 0 applies nothing: pass -1, listed first). */
int ql_plan_schedule(const ql_circuit* c, ql_dtype dtype, int32_t* pass_of_gate,
                     int32_t* order);

/* Algorithmic HBM bytes of the handle's plan in a mode (QL_MODE_*: reads +
 * writes of psi and lambda by the tile passes; 0 for a whole-state plan; a call
 * that the run kernel takes moves none). */
int ql_plan_state_bytes(const ql_circuit* c, ql_dtype dtype, int64_t batch, int mode,
                        double* out);

/* ---- timing (for benchmarks) --------------------------------------------- */

/* Kernel classes: 0 tile passes, 1 whole-state and run kernels, 2 angle binding and
 * embedding, 3 reductions. enable = 0 turns timing off; otherwise bit c of
 * enable selects class c (15: all). Every launch of a selected class is then
 * bracketed by HIP events on the call's stream (each pair costs host time,
 * which shows on launch-bound workloads: time only the classes needed).
 * ql_timing_read synchronises on the last event and returns the summed
 * milliseconds per class in ms[0..3] and the launch counts in
 * launches[0..3]. Reading resets them. Not thread-safe: one timed call in
 * flight per handle. */
int ql_timing_enable(ql_circuit* c, int enable);
int ql_timing_read(ql_circuit* c, double ms[4], int32_t launches[4]);

#ifdef __cplusplus
}
#endif

#endif /* QLAYER_H */
