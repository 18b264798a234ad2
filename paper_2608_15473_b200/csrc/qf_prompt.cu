// C ABI of the prompt side: placing packed tokens into the cache (qf_rope_append), attention over whole prompts
// (qf_prompt_attend) and the sweep of a prefix that requests share (qf_prefix_partial, qf_prefix_step).
// See include/qf.h for the contract.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "../../include/qf.h"
#include "../../include/qf_testing.h"
#include "qf_common.cuh"
#include "qf_host.h"
#include "qf_rope.cuh"
#include "qf_rows.cuh"

namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
bool misaligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// Positions and rows of the row kernels stay below this, so that their 32-bit arithmetic has room.
constexpr int kMostPositions = 1 << 30;

// A token row stride in elements: 0 = the packed width; rows must start on 16 bytes and not overlap.
bool bad_stride(int64_t stride, long long width) { return stride != 0 && (stride < width || (stride & 7)); }

template <bool PREFIX>
int launch_rows(const qf::RowsArgs &A, const qf::DevParams &P, const qf_params *p, char *ws, int sms, cudaStream_t st)
{
    if (p->flags & QF_FLAG_SIMPLE_KERNEL) {
        const long long units = (long long)A.total_rows * P.num_q_heads;
        const long long blocks = (units + qf::kRowsSimpleWarps - 1) / qf::kRowsSimpleWarps;
        if (blocks > 0x7fffffffll) return QF_ERR_UNSUPPORTED;
        qf::rows_simple_kernel<PREFIX, qf::kKvBf16><<<(unsigned)blocks, qf::kRowsSimpleWarps * 32, 0, st>>>(A, P, {});
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return qf_host::cuda_fail(e, "rows_simple_kernel launch");
        qf_host::set_launches(1);
        return QF_OK;
    }
    qf::RowsMaps maps;
    size_t len;
    char *msg = qf_host::cuda_msg(&len);
    if (qf::make_rows_maps(&maps, A, P, false, msg, len)) return QF_ERR_CUDA;
    cudaError_t e = qf::launch_rows_kernels<PREFIX, qf::kKvBf16>(maps, A, P, {}, ws, sms, st);
    if (e != cudaSuccess) return qf_host::cuda_fail(e, "rows_kernel launch");
    qf_host::set_launches(2);
    return QF_OK;
}

constexpr int kMostAxes = 8;

// The bf16 cache's placing kernel, for checked arguments.
int place(qf::RopeArgs &A, const qf::RopeAxes &X, const qf_params *p, int sms, void *cuda_stream)
{
    // one token per CTA until there are several for every SM, then steps of more: fewer, longer row lists per group
    A.tokens_per_cta = 1;
    while (A.tokens_per_cta < qf::kRopeMaxTokens && A.total_tokens >= 8 * A.tokens_per_cta * sms) A.tokens_per_cta *= 2;
    const long long steps = ((long long)A.total_tokens + A.tokens_per_cta - 1) / A.tokens_per_cta;
    const long long blocks = std::min<long long>(steps, (long long)qf::kRopeCtasPerSm * sms);
    const qf::DevParams P = qf_host::dev_params(p);
    cudaError_t e = X.positions ? qf::launch_rope<true>(A, X, P, (unsigned)blocks, (cudaStream_t)cuda_stream)
                                : qf::launch_rope<false>(A, {}, P, (unsigned)blocks, (cudaStream_t)cuda_stream);
    if (e != cudaSuccess) return qf_host::cuda_fail(e, "rope_append_kernel launch");
    qf_host::set_launches(1);
    return QF_OK;
}

}  // namespace

namespace qf_host {

int rope_args(qf::RopeArgs *out, qf::RopeAxes *axes, const void *q, const void *k, const void *v, void *q_out, void *k_out, void *k_cache,
              void *v_cache, const int32_t *block_table, const int32_t *cu_tokens, const int32_t *seq_lens,
              const int32_t *pos_base, const int32_t *positions, const int32_t *pair_axis, int num_axes, const void *q_gain,
              const void *k_gain, const float *inv_freq, const qf_params *p, const qf_rope_params *r, int *sms)
{
    set_launches(0);
    int rc = validate(p);
    if (rc != QF_OK) return rc;
    if (!r) return QF_ERR_NULL;
    if (r->total_tokens > kMostPositions) return QF_ERR_UNSUPPORTED;
    if (r->total_tokens <= 0 || r->rotary_dim < 0 || !(r->eps >= 0.f) || !std::isfinite(r->rot_scale)) return QF_ERR_BAD_SHAPE;
    if (r->rotary_dim > qf::kHeadDim || (r->rotary_dim & 15)) return QF_ERR_UNSUPPORTED;
    const long long D = qf::kHeadDim, Hq = p->num_q_heads, Hkv = p->num_kv_heads;
    if (bad_stride(r->q_stride, Hq * D) || bad_stride(r->k_stride, Hkv * D) || bad_stride(r->v_stride, Hkv * D))
        return QF_ERR_BAD_SHAPE;
    const bool cache = k_cache || v_cache;
    if (!cu_tokens || !seq_lens || (!q && !k) || (q && !q_out)) return QF_ERR_NULL;
    if (cache && (!k || !v || !k_cache || !v_cache)) return QF_ERR_NULL;      // the cache takes both or neither
    if (k && !cache && !k_out) return QF_ERR_NULL;                            // nowhere for the keys to go
    if (k_out && !k) return QF_ERR_NULL;
    if (r->rotary_dim > 0 && !inv_freq) return QF_ERR_NULL;
    if (positions) {
        if (r->rotary_dim > 0 && !pair_axis) return QF_ERR_NULL;
        if (num_axes <= 0) return QF_ERR_BAD_SHAPE;
        if (num_axes > kMostAxes) return QF_ERR_UNSUPPORTED;
    }
    for (const void *x : {q, k, v, (const void *)q_out, (const void *)k_out, (const void *)k_cache, (const void *)v_cache, q_gain, k_gain})
        if (misaligned(x, 16)) return QF_ERR_BAD_SHAPE;
    rc = check_device(sms);
    if (rc != QF_OK) return rc;
    qf::RopeArgs &A = *out;
    A.q = (const uint16_t *)q; A.k = (const uint16_t *)k; A.v = cache ? (const uint16_t *)v : nullptr;
    A.q_out = (uint16_t *)q_out; A.k_out = (uint16_t *)k_out;
    A.k_cache = (uint16_t *)k_cache; A.v_cache = (uint16_t *)v_cache;
    A.block_table = block_table; A.cu = cu_tokens; A.seq_lens = seq_lens; A.pos_base = pos_base;
    axes->positions = positions; axes->pair_axis = pair_axis; axes->num_axes = num_axes;
    A.q_gain = (const uint16_t *)q_gain; A.k_gain = (const uint16_t *)k_gain; A.inv_freq = inv_freq;
    A.q_stride = r->q_stride ? r->q_stride : Hq * D;
    A.k_stride = r->k_stride ? r->k_stride : Hkv * D;
    A.v_stride = r->v_stride ? r->v_stride : Hkv * D;
    A.total_tokens = r->total_tokens; A.rotary_dim = r->rotary_dim; A.interleaved = r->interleaved != 0;
    A.n_q = q ? (int)Hq : 0; A.n_k = k ? (int)Hkv : 0;
    A.rows = A.n_q + A.n_k + (cache ? (int)Hkv : 0);
    A.eps = r->eps; A.rot_scale = r->rot_scale;
    return QF_OK;
}

}  // namespace qf_host

extern "C" {

int qf_rope_frequencies(float *inv_freq, float *rot_scale, int rotary_dim, double theta, int scaling, double factor,
                        double original_len, double beta_fast, double beta_slow)
{
    if (!inv_freq || !rot_scale) return QF_ERR_NULL;
    if (rotary_dim <= 0 || !(theta > 1.0) || !std::isfinite(theta)) return QF_ERR_BAD_SHAPE;
    if (rotary_dim > qf::kHeadDim || (rotary_dim & 15)) return QF_ERR_UNSUPPORTED;
    if (scaling < QF_ROPE_PLAIN || scaling > QF_ROPE_YARN) return QF_ERR_UNSUPPORTED;
    if (scaling != QF_ROPE_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return QF_ERR_BAD_SHAPE;
    if (scaling == QF_ROPE_YARN && !(original_len > 0 && beta_slow > 0 && beta_fast > beta_slow)) return QF_ERR_BAD_SHAPE;
    const double d = rotary_dim;
    const double base = scaling == QF_ROPE_NTK ? theta * std::pow(factor, d / (d - 2.0)) : theta;
    double lo = 0, hi = 1;
    if (scaling == QF_ROPE_YARN) {
        // the pair whose wave turns `turns` times over the original length
        auto pair_of = [&](double turns) { return d * std::log(original_len / (turns * 6.283185307179586)) / (2.0 * std::log(theta)); };
        lo = std::max(std::floor(pair_of(beta_fast)), 0.0);
        hi = std::min(std::ceil(pair_of(beta_slow)), d - 1.0);
        if (hi <= lo) hi = lo + 0.001;
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / d);
        if (scaling == QF_ROPE_LINEAR) f /= factor;
        if (scaling == QF_ROPE_YARN) {
            const double slow = std::min(std::max((i - lo) / (hi - lo), 0.0), 1.0);   // 1: interpolated, 0: left alone
            f = f / factor * slow + f * (1.0 - slow);
        }
        inv_freq[i] = (float)f;
    }
    *rot_scale = scaling == QF_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return QF_OK;
}

int qf_rope_append(const void *q, const void *k, const void *v, void *q_out, void *k_out, void *k_cache, void *v_cache,
                   const int32_t *block_table, const int32_t *cu_tokens, const int32_t *seq_lens,
                   const int32_t *pos_base, const void *q_gain, const void *k_gain, const float *inv_freq,
                   const qf_params *p, const qf_rope_params *r, void *cuda_stream)
{
    qf::RopeArgs A = {};
    qf::RopeAxes X = {};
    int sms = 0;
    const int rc = qf_host::rope_args(&A, &X, q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, pos_base,
                                      nullptr, nullptr, 0, q_gain, k_gain, inv_freq, p, r, &sms);
    return rc != QF_OK ? rc : place(A, X, p, sms, cuda_stream);
}

int qf_rope_append_axes(const void *q, const void *k, const void *v, void *q_out, void *k_out, void *k_cache, void *v_cache,
                        const int32_t *block_table, const int32_t *cu_tokens, const int32_t *seq_lens,
                        const int32_t *positions, const int32_t *pair_axis, int num_axes, const void *q_gain,
                        const void *k_gain, const float *inv_freq, const qf_params *p, const qf_rope_params *r,
                        void *cuda_stream)
{
    if (!positions) {
        qf_host::set_launches(0);
        const int rc0 = qf_host::validate(p);
        return rc0 != QF_OK ? rc0 : QF_ERR_NULL;
    }
    qf::RopeArgs A = {};
    qf::RopeAxes X = {};
    int sms = 0;
    const int rc = qf_host::rope_args(&A, &X, q, k, v, q_out, k_out, k_cache, v_cache, block_table, cu_tokens, seq_lens, nullptr, positions,
                                      pair_axis, num_axes, q_gain, k_gain, inv_freq, p, r, &sms);
    return rc != QF_OK ? rc : place(A, X, p, sms, cuda_stream);
}

int qf_rope_pair_axes(int32_t *pair_axis, int rotary_dim, const int32_t *sections, int num_axes, int interleaved)
{
    if (!pair_axis || !sections) return QF_ERR_NULL;
    if (rotary_dim <= 0 || num_axes <= 0) return QF_ERR_BAD_SHAPE;
    if (rotary_dim > qf::kHeadDim || (rotary_dim & 15) || num_axes > kMostAxes) return QF_ERR_UNSUPPORTED;
    long long pairs = 0;
    for (int a = 0; a < num_axes; ++a) {
        if (sections[a] < 0) return QF_ERR_BAD_SHAPE;
        pairs += sections[a];
    }
    if (pairs != rotary_dim / 2) return QF_ERR_BAD_SHAPE;
    if (!interleaved) {
        int j = 0;
        for (int a = 0; a < num_axes; ++a)
            for (int i = 0; i < sections[a]; ++i) pair_axis[j++] = a;
        return QF_OK;
    }
    // axis a > 0 owns the pairs a, a + num_axes, ... as far as its section reaches; axis 0 owns the others
    for (int j = 0; j < pairs; ++j) {
        const int a = j % num_axes;
        pair_axis[j] = a > 0 && j / num_axes < sections[a] ? a : 0;
    }
    for (int a = 1; a < num_axes; ++a)
        if (sections[a] > 0 && (long long)(sections[a] - 1) * num_axes + a >= pairs) return QF_ERR_BAD_SHAPE;   // no room in turn
    return QF_OK;
}

size_t qf_prompt_workspace_bytes(const qf_params *p, int total_tokens)
{
    if (qf_host::validate(p) != QF_OK || total_tokens <= 0) return 0;
    return align256(qf::rows_layout().total);
}

}  // extern "C"

namespace qf_host {
int prompt(const void *q, const void *k_cache, const void *v_cache, const ScaledKv *scaled, const int32_t *block_table,
           const int32_t *cu_tokens, const int32_t *seq_lens, void *out, float *lse, const qf_params *p, int total_tokens,
           int64_t q_stride, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    set_launches(0);
    int rc = validate(p);
    if (rc != QF_OK) return rc;
    const long long width = (long long)p->num_q_heads * qf::kHeadDim;
    if (total_tokens <= 0 || bad_stride(q_stride, width)) return QF_ERR_BAD_SHAPE;
    if (total_tokens > kMostPositions) return QF_ERR_UNSUPPORTED;
    if (!q || !k_cache || !v_cache || !cu_tokens || !seq_lens || !out || !lse) return QF_ERR_NULL;
    if (scaled && (!scaled->k_scale || !scaled->v_scale)) return QF_ERR_NULL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < qf_prompt_workspace_bytes(p, total_tokens))
        return QF_ERR_WORKSPACE;
    if (misaligned(k_cache, 128) || misaligned(v_cache, 128) || misaligned(q, 16) || misaligned(out, 32)) return QF_ERR_BAD_SHAPE;
    if (scaled && (misaligned(scaled->k_scale, 4) || misaligned(scaled->v_scale, 4))) return QF_ERR_BAD_SHAPE;
    int sms = 0;
    rc = check_device(&sms);
    if (rc != QF_OK) return rc;
    const qf::DevParams P = dev_params(p);
    qf::RowsArgs A = {};
    A.q = (const uint16_t *)q; A.k_cache = k_cache; A.v_cache = v_cache;
    A.cu = cu_tokens; A.lens = seq_lens; A.table = block_table;
    A.out = (uint16_t *)out; A.lse = lse; A.status = (unsigned long long *)workspace;
    A.q_stride = q_stride ? q_stride : width;
    A.n_seq = p->batch; A.table_width = p->max_pages_per_req; A.max_tokens = std::min(P.max_tokens, kMostPositions); A.total_rows = total_tokens;
    if (scaled) return launch_rows_scaled(A, P, p, *scaled, (char *)workspace, sms, (cudaStream_t)cuda_stream);
    return launch_rows<false>(A, P, p, (char *)workspace, sms, (cudaStream_t)cuda_stream);
}
}  // namespace qf_host

extern "C" {

int qf_prompt_attend(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_table,
                     const int32_t *cu_tokens, const int32_t *seq_lens, void *out, float *lse, const qf_params *p,
                     int total_tokens, int64_t q_stride, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    return qf_host::prompt(q, k_cache, v_cache, nullptr, block_table, cu_tokens, seq_lens, out, lse, p, total_tokens, q_stride, workspace,
                           workspace_bytes, cuda_stream);
}

size_t qf_prefix_workspace_bytes(const qf_params *p)
{
    if (qf_host::validate(p) != QF_OK) return 0;
    return align256(qf::rows_layout().total) + align256(qf_workspace_bytes(p));
}

int qf_prefix_partial(const void *q, const void *k_cache, const void *v_cache, const int32_t *prefix_table,
                      const int32_t *prefix_lens, const int32_t *group_offsets, float *o_part, float *m_part,
                      float *lse_part, const qf_params *p, int num_groups, int max_prefix_pages, void *workspace,
                      size_t workspace_bytes, void *cuda_stream)
{
    qf_host::set_launches(0);
    int rc = qf_host::validate(p);
    if (rc != QF_OK) return rc;
    if (num_groups <= 0 || max_prefix_pages <= 0) return QF_ERR_BAD_SHAPE;
    if (num_groups > p->batch || (long long)max_prefix_pages * qf::kPageSize >= (1ll << 31)) return QF_ERR_UNSUPPORTED;
    if (!q || !k_cache || !v_cache || !prefix_lens || !group_offsets || !o_part || !m_part || !lse_part) return QF_ERR_NULL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < align256(qf::rows_layout().total)) return QF_ERR_WORKSPACE;
    if (misaligned(k_cache, 128) || misaligned(v_cache, 128) || misaligned(q, 16) || misaligned(o_part, 32)) return QF_ERR_BAD_SHAPE;
    int sms = 0;
    rc = qf_host::check_device(&sms);
    if (rc != QF_OK) return rc;
    const qf::DevParams P = qf_host::dev_params(p);
    qf::RowsArgs A = {};
    A.q = (const uint16_t *)q; A.k_cache = k_cache; A.v_cache = v_cache;
    A.cu = group_offsets; A.lens = prefix_lens; A.table = prefix_table;
    A.o_part = o_part; A.m_part = m_part; A.lse_part = lse_part; A.status = (unsigned long long *)workspace;
    A.q_stride = (long long)p->num_q_heads * qf::kHeadDim;
    A.n_seq = num_groups; A.table_width = max_prefix_pages;
    A.max_tokens = std::min(qf::max_row_tokens(max_prefix_pages), kMostPositions); A.total_rows = p->batch;
    A.out_shards = P.out_shards; A.slot = P.out_shard0;
    return launch_rows<true>(A, P, p, (char *)workspace, sms, (cudaStream_t)cuda_stream);
}

int qf_prefix_step(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_table,
                   const int32_t *seq_lens, const int32_t *shard_ranges, const int32_t *prefix_table,
                   const int32_t *prefix_lens, const int32_t *group_offsets, float *o_part, float *m_part,
                   float *lse_part, float *out, float *lse, const qf_params *p, int num_groups, int max_prefix_pages,
                   void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    qf_host::set_launches(0);
    int rc = qf_host::validate(p);
    if (rc != QF_OK) return rc;
    if (p->out_shards != 0) return QF_ERR_BAD_SHAPE;      // the step owns its shard table: the prefix, then S shards
    if (!seq_lens || !shard_ranges || !out || !lse) return QF_ERR_NULL;
    if (misaligned(out, 16)) return QF_ERR_BAD_SHAPE;
    if (!workspace || workspace_bytes < qf_prefix_workspace_bytes(p)) return QF_ERR_WORKSPACE;
    qf_params wide = *p, merge = *p;
    wide.out_shards = merge.max_shards = p->max_shards + 1;
    rc = qf_host::validate(&merge);
    if (rc != QF_OK) return rc;
    rc = qf_prefix_partial(q, k_cache, v_cache, prefix_table, prefix_lens, group_offsets, o_part, m_part, lse_part,
                           &wide, num_groups, max_prefix_pages, workspace, workspace_bytes, cuda_stream);
    if (rc != QF_OK) return rc;
    int launches = qf_last_launch_count();
    const size_t own = align256(qf::rows_layout().total);
    wide.out_shard_offset = 1;
    rc = qf_decode_partial(q, k_cache, v_cache, block_table, seq_lens, shard_ranges, o_part, m_part, lse_part, &wide,
                           (char *)workspace + own, workspace_bytes - own, cuda_stream);
    if (rc != QF_OK) return rc;
    launches += qf_last_launch_count();
    rc = qf_combine(o_part, lse_part, nullptr, out, lse, &merge, cuda_stream);
    if (rc == QF_OK) qf_host::set_launches(launches + qf_last_launch_count());
    return rc;
}

int qf_prompt_status(const void *workspace, int32_t *host_status, void *cuda_stream)
{
    if (!workspace || !host_status) return QF_ERR_NULL;
    unsigned long long word = 0;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaMemcpyAsync(&word, workspace, sizeof word, cudaMemcpyDeviceToHost, st);
    if (e != cudaSuccess) return qf_host::cuda_fail(e, "cudaMemcpyAsync");
    e = cudaMemsetAsync(const_cast<void *>(workspace), 0, sizeof word, st);   // read and clear
    if (e != cudaSuccess) return qf_host::cuda_fail(e, "cudaMemsetAsync");
    e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return qf_host::cuda_fail(e, "cudaStreamSynchronize");
    *host_status = ((word >> 8) == qf::kRowsStatusTag) ? (int32_t)(word & 0xffull) : 0;
    return QF_OK;
}

int qf_prefix_status(const void *workspace, const qf_params *p, int32_t *host_status, void *cuda_stream)
{
    int rc = qf_host::validate(p);
    if (rc != QF_OK) return rc;
    int32_t own = 0, sweep = 0;
    if (!workspace || !host_status) return QF_ERR_NULL;
    rc = qf_prompt_status(workspace, &own, cuda_stream);
    if (rc != QF_OK) return rc;
    rc = qf_read_status((const char *)workspace + align256(qf::rows_layout().total), &sweep, cuda_stream);
    if (rc == QF_OK) *host_status = own | sweep;
    return rc;
}

int qf_rows_schedule(int causal, const int32_t *offsets, const int32_t *lens, int n_seq, int group, int num_kv_heads,
                     int max_tokens, int total_rows, int n_ctas, int32_t *records, int capacity)
{
    if (!offsets || !lens || (capacity > 0 && !records)) return QF_ERR_NULL;
    if (n_seq < 1 || group < 1 || group > 8 || num_kv_heads < 1 || max_tokens < 1 || total_rows < 1 || n_ctas < 1 ||
        n_ctas > qf::kRowsMaxCtas || capacity < 0)
        return QF_ERR_BAD_SHAPE;
    auto first = [&](int s) { return std::min(std::max(offsets[s], 0), total_rows); };
    auto plan = [&](int s) {
        qf::SeqPlan q;
        q.n = std::max(std::min(offsets[s + 1], total_rows) - first(s), 0);
        q.off = std::min(std::max(lens[s], 0), max_tokens);
        q.len = causal ? (int)std::min((long long)q.off + q.n, (long long)max_tokens) : q.off;
        return q;
    };
    const qf::RowShape shape{causal != 0, qf::kRowTile / group, group};
    long long per_head = 0;
    for (int s = 0; s < n_seq; ++s) per_head += qf::seq_cost(plan(s), shape);
    const long long total = per_head * num_kv_heads;
    const int n = qf::slices_of(total, n_ctas);
    auto locate = [&](int c) {
        if (c == n) return qf::SlicePos{0, num_kv_heads, 0, 0};
        long long rest, before = 0;
        const int h = qf::head_of(qf::cut_at(total, n, c), per_head, rest);
        for (int s = 0; s < n_seq; ++s) {
            const long long cost = qf::seq_cost(plan(s), shape);
            if (rest >= before && rest < before + cost) return qf::locate_in_seq(plan(s), shape, s, h, rest - before);
            before += cost;
        }
        return qf::SlicePos{0, num_kv_heads, 0, 0};
    };
    int count = 0;
    for (int c = 0; total > 0 && c < n; ++c) {
        qf::SliceWalk<decltype(plan), decltype(first)> walk(plan, first, shape, locate(c), locate(c + 1), n_seq, num_kv_heads, c);
        qf::RowsBlock b;
        int nt = 0, tiles = 0;
        while (walk.next(b, nt)) {
            if (count < capacity) {
                const int32_t r[12] = {c, b.seq, b.head, b.row0, b.rows, b.t_lo, b.t_hi, b.slot, b.narrow, b.off + (causal ? b.i0 : 0), b.len, tiles};
                std::copy(r, r + 12, records + (size_t)count * 12);
            }
            tiles += b.t_hi - b.t_lo;
            ++count;
        }
    }
    return count;
}

}  // extern "C"
