// Process-wide switches for tests and measurements (not part of the public ABI of include/heta.h; the
// symbols are exported so that the Python tests can reach them).  Not thread-safe.
#pragma once

#include "heta.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 0 = by size (the default): a relation of at least 2^18 edges + rows is ingested by the per-relation device
 * kernels; the smaller relations of a graph together by the whole-block device ingest when their arrays lie on
 * the device or add up to 2^16 edges + rows, else on the host.  1 = everything on the host, 2 = everything by the
 * per-relation device kernels, 3 = small relations always by the whole-block device ingest.  All paths
 * produce identical index arrays. */
heta_status heta_ingest_force(int32_t mode);

/* When on, every projection runs the register-staged kernel that otherwise only serves operands whose
 * rows are not 16-byte aligned; off (the default) prefers the direct-to-LDS pipeline.  Results agree to
 * rounding order. */
heta_status heta_projection_force_staged(int32_t on);

/* fp32 x fp32 projections on the direct pipeline form every product from three bf16 terms per operand (six
 * bf16 MFMAs, fp32 accumulation: products exact to 2^-24).  When on, they run on the fp32 MFMA (32x32x2)
 * instead: the same results to rounding order at about 2.5 times the matrix-pipe time. */
heta_status heta_projection_f32_native(int32_t on);

/* Workspaces of handles that are to grow beyond `bytes` fail to (HETA_ERR_OOM), as with a device that is full; what a handle
 * holds already stays usable.  0 (the default): no limit. */
heta_status heta_workspace_limit(int64_t bytes);

/* How heta_linear_xent (backward = 0) and heta_linear_xent_bwd read bf16 operands at these addresses, of the arguments' sizes; no device call.  out, int64 [8]: 1 where W and where
 * in are copied to aligned rows first; 1 where the operands of the logits, of grad_in and of grad_W go straight into LDS; the classes of a piece, which a copy of W holds;
 * and the largest offset in bytes that such loads make from a tile's first row, of W and of in, which have 32 bits for it. */
heta_status heta_xent_reads(const heta_linear_xent_bwd_args *args, int32_t backward, int64_t *out);

#ifdef __cplusplus
}
#endif
