// C ABI of the scaled cache: keys and values held in one byte each, with a scale per page and KV head.  Placing
// (qf_rope_append_scaled), the decode sweep and step (qf_decode_partial_scaled, qf_decode_step_scaled) and attention of
// prompts (qf_prompt_attend_scaled).  See include/qf.h for the contract.
#include <cuda_runtime.h>

#include <algorithm>

#include "../../include/qf.h"
#include "qf_common.cuh"
#include "qf_host.h"
#include "qf_place_scaled.cuh"
#include "qf_rows.cuh"
#include "qf_simple.cuh"
#include "qf_sweep.cuh"

namespace {

bool misaligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
bool known_type(int kv_type) { return kv_type == QF_KV_E4M3 || kv_type == QF_KV_INT8; }
// Parameters that are wrong in themselves come first, as in every call.
int refuse(const qf_params *p, int code)
{
    qf_host::set_launches(0);
    const int rc = qf_host::validate(p);
    return rc != QF_OK ? rc : code;
}
static_assert((int)QF_KV_E4M3 == (int)qf::kKvE4m3 && (int)QF_KV_INT8 == (int)qf::kKvInt8, "the header's types are the kernels'");

template <int KV, int G>
void launch_simple_g(const void *q, const void *k, const void *v, const qf_host::ScaledKv &s, const int32_t *bt, const int32_t *sl,
                     const int32_t *sr, float *o, float *m, float *l, const qf::DevParams &P, unsigned long long *header,
                     unsigned long long epoch, cudaStream_t st)
{
    if (P.group != G) {
        if constexpr (G > 1) launch_simple_g<KV, G - 1>(q, k, v, s, bt, sl, sr, o, m, l, P, header, epoch, st);
        return;
    }
    dim3 grid(P.max_shards, P.num_kv_heads, P.batch);
    qf::sweep_simple_kernel<G, KV><<<grid, qf::kSimpleWarps * 32, 0, st>>>((const uint16_t *)q, k, v, s.k_scale, s.v_scale, bt, sl, sr,
                                                                          o, m, l, P, header, epoch);
}

}  // namespace

namespace qf_host {

int launch_simple_scaled(const void *q, const void *k, const void *v, const ScaledKv &s, const int32_t *bt, const int32_t *sl,
                         const int32_t *sr, float *o, float *m, float *l, const qf::DevParams &P, unsigned long long *header,
                         unsigned long long epoch, cudaStream_t st)
{
    if (s.kind == qf::kKvE4m3) launch_simple_g<qf::kKvE4m3, 8>(q, k, v, s, bt, sl, sr, o, m, l, P, header, epoch, st);
    else launch_simple_g<qf::kKvInt8, 8>(q, k, v, s, bt, sl, sr, o, m, l, P, header, epoch, st);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? QF_OK : cuda_fail(e, "sweep_simple_kernel launch");
}

int launch_sweep_scaled(const void *q, const void *k, const void *v, const ScaledKv &s, const int32_t *bt, const int32_t *sl,
                        const int32_t *sr, float *o, float *m, float *l, const qf::DevParams &P, char *ws,
                        const qf::WorkspaceLayout &wsl, int n_ctas, unsigned long long epoch, cudaStream_t st, cudaEvent_t ev0,
                        cudaEvent_t ev1, char *msg, size_t msg_len, int *launches, bool skip_finish)
{
    CUtensorMap kmap, vmap;
    if (qf::make_scaled_map(&kmap, k, P.num_pages, P.num_kv_heads, P.kv_nhd != 0, true, msg, msg_len)) return QF_ERR_CUDA;
    if (qf::make_scaled_map(&vmap, v, P.num_pages, P.num_kv_heads, P.kv_nhd != 0, true, msg, msg_len)) return QF_ERR_CUDA;
    return s.kind == qf::kKvE4m3
               ? qf::launch_sweep_kv<qf::kKvE4m3>(kmap, vmap, {s.k_scale, s.v_scale}, q, bt, sl, sr, o, m, l, P, ws, wsl, n_ctas, epoch, st, ev0,
                                                  ev1, msg, msg_len, launches, skip_finish)
               : qf::launch_sweep_kv<qf::kKvInt8>(kmap, vmap, {s.k_scale, s.v_scale}, q, bt, sl, sr, o, m, l, P, ws, wsl, n_ctas, epoch, st, ev0,
                                                  ev1, msg, msg_len, launches, skip_finish);
}

int launch_rows_scaled(const qf::RowsArgs &A, const qf::DevParams &P, const qf_params *p, const ScaledKv &s, char *ws, int sms, cudaStream_t st)
{
    const bool e4m3 = s.kind == qf::kKvE4m3;
    if (p->flags & QF_FLAG_SIMPLE_KERNEL) {
        const long long units = (long long)A.total_rows * P.num_q_heads;
        const long long blocks = (units + qf::kRowsSimpleWarps - 1) / qf::kRowsSimpleWarps;
        if (blocks > 0x7fffffffll) return QF_ERR_UNSUPPORTED;
        if (e4m3) qf::rows_simple_kernel<false, qf::kKvE4m3><<<(unsigned)blocks, qf::kRowsSimpleWarps * 32, 0, st>>>(A, P, {s.k_scale, s.v_scale});
        else qf::rows_simple_kernel<false, qf::kKvInt8><<<(unsigned)blocks, qf::kRowsSimpleWarps * 32, 0, st>>>(A, P, {s.k_scale, s.v_scale});
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return cuda_fail(e, "rows_simple_kernel launch");
        set_launches(1);
        return QF_OK;
    }
    qf::RowsMaps maps;
    size_t len;
    char *msg = cuda_msg(&len);
    if (qf::make_rows_maps(&maps, A, P, true, msg, len)) return QF_ERR_CUDA;
    const cudaError_t e = e4m3 ? qf::launch_rows_kernels<false, qf::kKvE4m3>(maps, A, P, {s.k_scale, s.v_scale}, ws, sms, st)
                               : qf::launch_rows_kernels<false, qf::kKvInt8>(maps, A, P, {s.k_scale, s.v_scale}, ws, sms, st);
    if (e != cudaSuccess) return cuda_fail(e, "rows_kernel launch");
    set_launches(2);
    return QF_OK;
}

}  // namespace qf_host

extern "C" {

int qf_rope_append_scaled(const void *q, const void *k, const void *v, void *q_out, void *k_out, void *k_cache, void *v_cache,
                          float *k_scale, float *v_scale, const int32_t *block_table, const int32_t *cu_tokens,
                          const int32_t *seq_lens, const int32_t *pos_base, const int32_t *positions, const int32_t *pair_axis,
                          int num_axes, const void *q_gain, const void *k_gain, const float *inv_freq, int kv_type,
                          const qf_params *p, const qf_rope_params *r, void *cuda_stream)
{
    if (!known_type(kv_type)) return refuse(p, QF_ERR_UNSUPPORTED);
    if ((k_cache || v_cache) && (!k_scale || !v_scale)) return refuse(p, QF_ERR_NULL);
    if (misaligned(k_scale, 4) || misaligned(v_scale, 4)) return refuse(p, QF_ERR_BAD_SHAPE);
    qf::RopeArgs A = {};
    qf::RopeAxes X = {};
    int sms = 0;
    const int rc = qf_host::rope_args(&A, &X, q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, pos_base, positions,
                                      pair_axis, num_axes, q_gain, k_gain, inv_freq, p, r, &sms);
    if (rc != QF_OK) return rc;
    const qf::DevParams P = qf_host::dev_params(p);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = kv_type == QF_KV_E4M3 ? qf::launch_place_scaled<qf::kKvE4m3>(A, X, k_scale, v_scale, P, sms, st)
                                                : qf::launch_place_scaled<qf::kKvInt8>(A, X, k_scale, v_scale, P, sms, st);
    if (e != cudaSuccess) return qf_host::cuda_fail(e, "place_scaled_kernel launch");
    qf_host::set_launches(1);
    return QF_OK;
}

int qf_decode_partial_scaled(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale,
                             const int32_t *block_table, const int32_t *seq_lens, const int32_t *shard_ranges, float *o_part,
                             float *m_part, float *lse_part, int kv_type, const qf_params *p, void *workspace,
                             size_t workspace_bytes, void *cuda_stream)
{
    if (!known_type(kv_type)) return refuse(p, QF_ERR_UNSUPPORTED);
    const qf_host::ScaledKv s{kv_type, k_scale, v_scale};
    return qf_host::sweep(q, k_cache, v_cache, &s, block_table, seq_lens, shard_ranges, nullptr, o_part, m_part, lse_part, nullptr,
                          nullptr, nullptr, p, workspace, workspace_bytes, cuda_stream);
}

int qf_decode_step_scaled(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale,
                          const int32_t *block_table, const int32_t *seq_lens, const int32_t *shard_ranges,
                          const int32_t *shard_counts, float *o_part, float *m_part, float *lse_part, float *out, float *lse,
                          int kv_type, const qf_params *p, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (!known_type(kv_type)) return refuse(p, QF_ERR_UNSUPPORTED);
    const qf_host::ScaledKv s{kv_type, k_scale, v_scale};
    return qf_host::step(q, k_cache, v_cache, &s, block_table, seq_lens, shard_ranges, shard_counts, o_part, m_part, lse_part, out, lse,
                         p, workspace, workspace_bytes, cuda_stream);
}

int qf_prompt_attend_scaled(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale,
                            const int32_t *block_table, const int32_t *cu_tokens, const int32_t *seq_lens, void *out, float *lse,
                            int kv_type, const qf_params *p, int total_tokens, int64_t q_stride, void *workspace,
                            size_t workspace_bytes, void *cuda_stream)
{
    if (!known_type(kv_type)) return refuse(p, QF_ERR_UNSUPPORTED);
    const qf_host::ScaledKv s{kv_type, k_scale, v_scale};
    return qf_host::prompt(q, k_cache, v_cache, &s, block_table, cu_tokens, seq_lens, out, lse, p, total_tokens, q_stride, workspace,
                           workspace_bytes, cuda_stream);
}

}  // extern "C"
