// Host-side helpers of the C boundary shared by its translation units (defined in qf_api.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

#include "../../include/qf.h"
#include "qf_common.cuh"

namespace qf { struct RopeArgs; struct RopeAxes; struct RowsArgs; struct WorkspaceLayout; }

namespace qf_host {

int validate(const qf_params *p);                        // QF_OK or the error code of these parameters
qf::DevParams dev_params(const qf_params *p);
int check_device(int *sm_count);                         // the current device is a compute-capability 10.x part
int cuda_fail(cudaError_t e, const char *what);          // records the text, returns QF_ERR_CUDA
char *cuda_msg(size_t *len);                             // the buffer qf_strerror(QF_ERR_CUDA) reads
void set_launches(int n);                                // what qf_last_launch_count reports
// The checks that the placing calls share, and their kernels' arguments.
int rope_args(qf::RopeArgs *out, qf::RopeAxes *axes, const void *q, const void *k, const void *v, void *q_out, void *k_out, void *k_cache,
              void *v_cache, const int32_t *block_table, const int32_t *cu_tokens, const int32_t *seq_lens,
              const int32_t *pos_base, const int32_t *positions, const int32_t *pair_axis, int num_axes, const void *q_gain,
              const void *k_gain, const float *inv_freq, const qf_params *p, const qf_rope_params *r, int *sms);

// A cache of one byte per number (qf_scaled.cu); kind: qf::kKvE4m3 or qf::kKvInt8.
struct ScaledKv { int kind; const float *k_scale, *v_scale; };
// The sweep and the step behind qf_decode_partial and qf_decode_step, for either kind of cache (scaled: null = bf16).
int sweep(const void *q, const void *k_cache, const void *v_cache, const ScaledKv *scaled, const int32_t *block_table,
          const int32_t *seq_lens, const int32_t *shard_ranges, const int32_t *shard_counts, float *o_part, float *m_part,
          float *lse_part, float *step_out, float *step_lse, bool *merged, const qf_params *p, void *workspace,
          size_t workspace_bytes, void *cuda_stream);
int step(const void *q, const void *k_cache, const void *v_cache, const ScaledKv *scaled, const int32_t *block_table,
         const int32_t *seq_lens, const int32_t *shard_ranges, const int32_t *shard_counts, float *o_part, float *m_part,
         float *lse_part, float *out, float *lse, const qf_params *p, void *workspace, size_t workspace_bytes, void *cuda_stream);

int prompt(const void *q, const void *k_cache, const void *v_cache, const ScaledKv *scaled, const int32_t *block_table,
           const int32_t *cu_tokens, const int32_t *seq_lens, void *out, float *lse, const qf_params *p, int total_tokens,
           int64_t q_stride, void *workspace, size_t workspace_bytes, void *cuda_stream);
int launch_rows_scaled(const qf::RowsArgs &A, const qf::DevParams &P, const qf_params *p, const ScaledKv &s, char *ws, int sms, cudaStream_t st);
int launch_simple_scaled(const void *q, const void *k, const void *v, const ScaledKv &s, const int32_t *bt, const int32_t *sl,
                         const int32_t *sr, float *o, float *m, float *l, const qf::DevParams &P, unsigned long long *header,
                         unsigned long long epoch, cudaStream_t st);
int launch_sweep_scaled(const void *q, const void *k, const void *v, const ScaledKv &s, const int32_t *bt, const int32_t *sl,
                        const int32_t *sr, float *o, float *m, float *l, const qf::DevParams &P, char *ws,
                        const qf::WorkspaceLayout &wsl, int n_ctas, unsigned long long epoch, cudaStream_t st, cudaEvent_t ev0,
                        cudaEvent_t ev1, char *msg, size_t msg_len, int *launches, bool skip_finish);

}  // namespace qf_host
