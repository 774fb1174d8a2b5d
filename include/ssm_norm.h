/*
 * ssm_norm.h -- C ABI of the norm in front of a block, with its residual add (Section 3.4: the block is repeated, interleaved
 * with standard normalization and residual connections).  A neighbour of the hot path, not part of the scan itself.
 *
 * Per row of D elements:
 *     s = x + residual   rounded once to residual_dtype          (SSM_NORM_FLAG_HAS_RESIDUAL; otherwise s = x)
 *     m = mean(s),  r = 1 / sqrt(mean((s - m)^2) + eps)           (SSM_NORM_FLAG_RMS: m = 0)
 *     y = (s - m) r * weight + bias                               (bias: SSM_NORM_FLAG_HAS_BIAS)
 * The norm is of the rounded s, which is what residual_out holds and the backward call is given.
 * Backward for loss = sum(dy * y) + sum(dresidual_out * s), with xh = (s - m) r and q = dy * weight:
 *     ds = r (q - mean(q) - xh mean(q xh)) + dresidual_out         (SSM_NORM_FLAG_RMS: without mean(q))
 *     dx = ds in io_dtype, dresidual = ds in residual_dtype;  dweight = sum_rows dy xh;  dbias = sum_rows dy
 *
 * Conventions as in ssm_scan.h: plain C; every pointer but `p` is caller-owned DEVICE memory valid for `stream` on the
 * current device; the library allocates nothing; calls enqueue and return; argument errors are reported before anything is
 * launched; outputs are overwritten; inputs must not alias outputs; results are bitwise reproducible for the same problem and
 * pointers' alignment (fixed summation orders, no atomics).  Layouts: x, y, dy, dx dense [rows][D] io_dtype; residual,
 * residual_out, dresidual_out, dresidual dense [rows][D] residual_dtype; s is residual_out, or x where there is no residual;
 * weight, bias, dweight, dbias float32 [D]; stats float32 [rows][2] (m, r).  Arithmetic and sums are float32.  Every
 * pointer is aligned to its element; rows of whole 16 bytes at aligned pointers (to 16 bytes, float32 ones beside bf16 io to 32)
 * take wide accesses, bf16 rows of whole pairs (4 and 8 bytes) narrower ones.
 * NaN and Inf propagate within their row (and into dweight and dbias).  The backward call waits for its own copies of long rows, for
 * a limited time; a wait that runs out (a fault elsewhere) leaves NaN in the row, in those after it, in dweight and in dbias.
 */
#ifndef SSM_NORM_H_
#define SSM_NORM_H_

#include "ssm_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
  SSM_NORM_FLAG_RMS = 1u,          /* no mean is subtracted                                     */
  SSM_NORM_FLAG_HAS_BIAS = 2u,     /* bias is given; otherwise 0 and dbias not produced         */
  SSM_NORM_FLAG_HAS_RESIDUAL = 4u, /* residual is given                                         */
  SSM_NORM_FLAG_TEST_WITHHOLD = 16u /* test hook for the bounded waits of backward: where rows come by copies that are waited
                                      for, one stays away, so that the waits run out (at once) */
};

typedef struct {
  int64_t rows;            /* 1 .. 2^31 - 1 */
  int32_t D;               /* 1 .. 2^28 */
  int32_t io_dtype;        /* ssm_dtype_t */
  int32_t residual_dtype;  /* ssm_dtype_t: io_dtype or SSM_F32; io_dtype where there is no residual */
  uint32_t flags;          /* SSM_NORM_FLAG_* */
  float eps;               /* >= 0 and finite */
} ssm_norm_problem_t;

/*
 * Forward.  x, weight, y required; residual required iff SSM_NORM_FLAG_HAS_RESIDUAL (else NULL), bias iff
 * SSM_NORM_FLAG_HAS_BIAS (else NULL); residual_out may be NULL (not wanted) and is NULL without a residual; stats may be NULL
 * (not wanted; the backward call needs them).
 */
SSM_API ssm_status_t ssm_norm_fwd(const ssm_norm_problem_t* p, const void* x, const void* residual, const float* weight,
                                  const float* bias, void* y, void* residual_out, float* stats,
                                  void* stream /* cudaStream_t */);

/* Bytes of scratch ssm_norm_bwd needs (partial sums of dweight and dbias); 0 for an invalid problem. */
SSM_API size_t ssm_norm_bwd_workspace_bytes(const ssm_norm_problem_t* p);

/*
 * Backward.  s, weight, dy, stats, dx, dweight required; dresidual_out (only with a residual) may be NULL: nothing arrives
 * there; dresidual may be NULL, and is NULL where residual_dtype is io_dtype: dx is the gradient of both then; dbias required
 * iff SSM_NORM_FLAG_HAS_BIAS (else NULL).  eps is not used.  workspace of at least ssm_norm_bwd_workspace_bytes(p) bytes,
 * 16-byte aligned; contents undefined between calls; calls that overlap on the GPU must not share it.
 */
SSM_API ssm_status_t ssm_norm_bwd(const ssm_norm_problem_t* p, const void* s, const float* weight, const void* dy,
                                  const float* stats, const void* dresidual_out, void* dx, void* dresidual,
                                  float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                                  void* stream /* cudaStream_t */);

#ifdef __cplusplus
}
#endif
#endif /* SSM_NORM_H_ */
