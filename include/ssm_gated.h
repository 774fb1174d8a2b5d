/*
 * ssm_gated.h -- C ABI of the gated linear recurrence: the recurrence beside the selective scan whose state is one value
 * per channel and whose retention is itself a gate.
 *
 * Per batch b and channel d independently, with the state h[b,d] and t = 1..L:
 *     h[t] = a[t] * h[t-1] + u[t],   y[b,t,d] = h[t]
 * in one of two forms, sigma being the logistic function:
 *   convex (Theorem 1 of Section 3.5.1: what the selective scan becomes for N = 1, A = -1, B = 1):
 *     g = sigma(gate[b,t,d]);            a = 1 - g;           u = g * x[b,t,d]
 *   decay (SSM_GATED_FLAG_DECAY: a parameter A[d] <= 0 per channel, the gate as the step size of A-bar = exp(delta A) of
 *   Eq. 4, and a gate on the input, scaled so that an input of unit variance gives a state of unit variance):
 *     rho = sigma(gate[b,t,d]);  a = exp(rho * A[d]);  u = sqrt(1 - a^2) * sigma(in_gate[b,t,d]) * x[b,t,d]
 * reset (optional): where reset[b,t] != 0, h[t-1] is taken as zero whatever it holds, so that sequences that lie one behind
 * the other in a row do not see each other (for t = 1 this means h0).
 * Backward for loss = sum(dy * y) + sum(dh_last * h[L]):
 *     mu[t] = dy[t] + a[t+1] mu[t+1]     (mu[L] = dy[L] + dh_last; nothing arrives from a step t+1 that resets)
 *     convex:  dx = mu g;   dgate = mu (x - h[t-1]) g (1 - g)
 *     decay:   with beta = sqrt(1 - a^2), iota = sigma(in_gate), m = mu (a h[t-1] - a^2 iota x / beta):
 *              dx = mu beta iota;  din_gate = mu beta x iota (1 - iota);  dgate = m A rho (1 - rho);  dA = sum_{b,t} m rho
 *     dh0 = a[1] mu[1]                    (h[t-1] = 0 where step t resets)
 *
 * Conventions as in ssm_scan.h: plain C; every pointer but `p` is caller-owned DEVICE memory valid for `stream` on the
 * current device; the library allocates nothing; calls enqueue and return; argument errors are reported before anything is
 * launched; outputs are overwritten; inputs must not alias outputs.
 *   - x, gate, in_gate, dx, dgate, din_gate: [batch][L] rows of D io_dtype elements.  The rows of each lie ld_* elements
 *     apart (0: D, one behind the other), as column ranges of one projection do; the rows of a batch entry follow those of the
 *     one before it at the same distance.  A distance below D or above 2^28 is refused.  What lies between the rows is neither read nor
 *     written.  y, dy: dense [batch][L][D] io_dtype.
 *   - A, dA float32 [D]; h0, h_last, dh_last, dh0 and the h of ssm_gated_step float32 [batch][D]; reset one byte per step,
 *     [batch][L] (ssm_gated_step: [batch]).
 *   - Arithmetic, states and sums are float32; y and the gradients of the inputs are rounded once to io_dtype.  (Decay
 *     form: an in_gate below -44, which lets less than 1e-19 of its input through, may let nothing through in the forward pass and
 *     the step.  The gradients of gates are good relative to their own size however far the gates are open.)
 *   - Every pointer is aligned to its element.  Rows that begin and end on 16 bytes take the widest copies, such on 4 bytes
 *     narrower ones, others single elements, each slower than the one before.  bf16 pairs of channels also want A, h0, h_last,
 *     dh_last, dh0 and the saved states aligned to 8 bytes; otherwise single elements move.
 *   - Results are bitwise reproducible for the same problem, pointers' alignment and presence of optional arguments.
 *   - The blocks that share a channel's sequence wait for one another, for a limited time.  A wait that runs out (a fault
 *     elsewhere) leaves NaN in what its block writes from there on, h_last, dh0 and its share of dA included (not in steps that a
 *     reset within the same tile cuts off).
 *   - NaN and Inf propagate along the recurrence (and not across a reset).  A > 0 is not validated and gives NaN.
 */
#ifndef SSM_GATED_H_
#define SSM_GATED_H_

#include "ssm_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
  SSM_GATED_FLAG_DECAY = 1u,       /* the decay form: A and in_gate are given                                          */
  SSM_GATED_FLAG_SAVE_STATES = 4u, /* forward: also write the states that backward restarts from; backward: they are
                                      given (otherwise the call rebuilds them in its workspace)                       */
  SSM_GATED_FLAG_TEST_WITHHOLD = 16u /* test hook for the bounded waits: where blocks exchange, one sends nothing, so that
                                      the others' waits run out (at once)                                             */
};

typedef struct {
  int32_t batch, L, D;   /* all >= 1; D at most 2^28, batch * L below 2^31, batch * ceil(D / 32) below 2^27, L below 2^31 - 2^16 */
  int32_t io_dtype;      /* ssm_dtype_t */
  uint32_t flags;        /* SSM_GATED_FLAG_* */
  int64_t ld_x, ld_gate, ld_in_gate;      /* distance of rows in elements; 0: D.  Other than 0 only where it is used   */
  int64_t ld_dx, ld_dgate, ld_din_gate;
} ssm_gated_problem_t;

/* Bytes of the `saved_states` buffer: float32, opaque, valid for backward calls of the same batch, L, D and form on the same
 * inputs.  0 for an invalid problem. */
SSM_API size_t ssm_gated_saved_state_bytes(const ssm_gated_problem_t* p);

/*
 * Forward.  x, gate, y required; in_gate and A required iff SSM_GATED_FLAG_DECAY (else NULL); reset, h0, h_last may be NULL
 * (no reset; zero; not wanted); saved_states required iff SSM_GATED_FLAG_SAVE_STATES (else NULL).  Needs no workspace.
 */
SSM_API ssm_status_t ssm_gated_fwd(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate,
                                   const float* A, const uint8_t* reset, const float* h0, void* y, float* h_last,
                                   float* saved_states, void* stream /* cudaStream_t */);

/* Bytes of scratch ssm_gated_bwd needs (0 is possible, and stands for an invalid problem too). */
SSM_API size_t ssm_gated_bwd_workspace_bytes(const ssm_gated_problem_t* p);

/*
 * Backward.  x, gate, in_gate, A, reset, h0 as in the forward call; dy, dx, dgate required; din_gate and dA required iff
 * SSM_GATED_FLAG_DECAY (else NULL); dh_last, dh0 may be NULL; saved_states of the forward call iff
 * SSM_GATED_FLAG_SAVE_STATES (else NULL).  workspace of at least ssm_gated_bwd_workspace_bytes(p) bytes, 16-byte aligned
 * (NULL where that is 0); contents undefined between calls; calls that overlap on the GPU must not share it.
 */
SSM_API ssm_status_t ssm_gated_bwd(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate,
                                   const float* A, const uint8_t* reset, const float* h0, const void* dy,
                                   const float* dh_last, const float* saved_states, void* dx, void* dgate, void* din_gate,
                                   float* dA, float* dh0, void* workspace, size_t workspace_bytes,
                                   void* stream /* cudaStream_t */);

/*
 * One step of decoding: x, gate, in_gate and y hold one row per batch entry, h [batch][D] is updated in place.  p->L must be
 * 1; in_gate and A as in the forward call; reset [batch] may be NULL.  Flags other than SSM_GATED_FLAG_DECAY are refused.
 */
SSM_API ssm_status_t ssm_gated_step(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate,
                                    const float* A, const uint8_t* reset, float* h, void* y,
                                    void* stream /* cudaStream_t */);

#ifdef __cplusplus
}
#endif
#endif /* SSM_GATED_H_ */
