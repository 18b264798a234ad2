// Attention of packed query rows over a paged cache: the problem's description, shared by both kernels, and the
// plain-load kernel (a validation aid selected by QF_FLAG_SIMPLE_KERNEL, as for the decode sweep).
//
// A sequence s owns the query rows cu[s] .. cu[s+1]-1 (tokens of a prompt, or requests that share a prefix) and
// a row of the page table.  Row i of it attends the positions below
//     prompt:  min(lens[s] + i + 1, max_tokens)        (causal: what was cached before, and itself)
//     prefix:  min(lens[s], max_tokens)                (every request sees the whole prefix).
#pragma once

#include "qf_common.cuh"
#include "qf_page_math.cuh"

namespace qf {

struct RowsArgs {
    const uint16_t *q;               // row r, query head h: q + r * q_stride + h * 128
    const uint16_t *k_cache, *v_cache;
    const int *cu, *lens, *table;    // [n_seq + 1], [n_seq], [n_seq, table_width] (nullptr: identity)
    uint16_t *out;                   // prompt: [rows, Hq, 128] bf16
    float *lse;                      // prompt: [rows, Hq]
    float *o_part, *m_part, *lse_part;   // prefix: slot `slot` of [rows, out_shards, Hq, (128)]
    unsigned long long *status;      // sticky tagged word (rows_status_or)
    long long q_stride;
    int n_seq, table_width, max_tokens, total_rows;
    int out_shards, slot;
};

// The status word of these operators is sticky, like the projection pair's: bits stay until the host has read
// them, and a word without the tag (fresh workspace) reads as clean.
constexpr unsigned long long kRowsStatusTag = 0x3A9D40B7E21C55ull;   // 56 bits
__device__ __forceinline__ void rows_status_or(unsigned long long *w, unsigned bits)
{
    unsigned long long old = *reinterpret_cast<volatile unsigned long long *>(w);
    for (int tries = 0; tries < (1 << 12); ++tries) {
        const unsigned long long cur = ((old >> 8) == kRowsStatusTag) ? (old & 0xffull) : 0ull;
        const unsigned long long prev = atomicCAS(w, old, (kRowsStatusTag << 8) | cur | bits);
        if (prev == old) return;
        old = prev;
    }
}

struct SeqRows { int first, n, off, len; };   // first row, rows, positions before row 0 (causal), positions in all
template <bool PREFIX>
__device__ __forceinline__ SeqRows seq_rows(const RowsArgs &A, int s)
{
    SeqRows r;
    r.first = min(max(A.cu[s], 0), A.total_rows);
    r.n = max(min(A.cu[s + 1], A.total_rows) - r.first, 0);
    const int cached = min(max(A.lens[s], 0), A.max_tokens);
    r.off = cached;
    r.len = PREFIX ? cached : (int)min((long long)cached + r.n, (long long)A.max_tokens);
    return r;
}
template <bool PREFIX>
__device__ __forceinline__ int row_limit(const SeqRows &r, int i)
{
    return PREFIX ? r.len : (int)min((long long)r.off + i + 1, (long long)r.len);
}

// Rows of the sequence would see positions beyond the table row (or the caller's bound): clamped, and reported if asked for.
template <bool PREFIX>
__device__ __forceinline__ bool seq_overruns(const RowsArgs &A, int s)
{
    const SeqRows r = seq_rows<PREFIX>(A, s);
    return r.n > 0 && (long long)max(A.lens[s], 0) + (PREFIX ? 0 : r.n) > A.max_tokens;
}

constexpr int kRowsSimpleWarps = 8;

// One warp per (row, query head), lane owns four channels, fp32 online softmax over the positions in order.
template <bool PREFIX>
__global__ void __launch_bounds__(kRowsSimpleWarps * 32)
rows_simple_kernel(RowsArgs A, DevParams P)
{
    const int Hq = P.num_q_heads, lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * kRowsSimpleWarps + (threadIdx.x >> 5);
    if (unit >= (long long)A.total_rows * Hq) return;
    const int row = (int)(unit / Hq), h = (int)(unit - (long long)row * Hq), c = h / P.group;
    // the last sequence whose first row is not behind this one (empty sequences share a boundary with it)
    int s = -1;
    if (A.n_seq > 0 && row >= A.cu[0] && row < A.cu[A.n_seq]) {
        int lo = 0, hi = A.n_seq;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (A.cu[mid] <= row) lo = mid; else hi = mid;
        }
        s = lo;
    }
    if (s < 0 && !PREFIX) return;                 // a row of no sequence is left as it was
    int limit = 0;
    if (s >= 0) {
        const SeqRows sr = seq_rows<PREFIX>(A, s);
        limit = row_limit<PREFIX>(sr, row - sr.first);
        if (P.check_bounds && row == sr.first && h == 0 && lane == 0 && seq_overruns<PREFIX>(A, s)) rows_status_or(A.status, kStatusBadPage);
    }
    const uint2 qw = *reinterpret_cast<const uint2 *>(A.q + (long long)row * A.q_stride + h * kHeadDim + lane * 4);
    float m = neg_inf(), l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < limit; ++i) {
        const long long at = (long long)s * A.table_width + (i >> 4);
        const long long phys = A.table ? (long long)A.table[at] : at;
        if (phys < 0 || phys >= P.num_pages) {    // a bad entry's tokens contribute nothing
            if (P.check_bounds && lane == 0) rows_status_or(A.status, kStatusBadPage);
            continue;
        }
        const size_t off = kv_row_offset(P, phys, c, i & 15) + lane * 4;
        const uint2 kw = *reinterpret_cast<const uint2 *>(A.k_cache + off);
        const uint2 vw = *reinterpret_cast<const uint2 *>(A.v_cache + off);
        float d = bf16lo_to_f32(qw.x) * bf16lo_to_f32(kw.x);
        d = fmaf(bf16hi_to_f32(qw.x), bf16hi_to_f32(kw.x), d);
        d = fmaf(bf16lo_to_f32(qw.y), bf16lo_to_f32(kw.y), d);
        d = fmaf(bf16hi_to_f32(qw.y), bf16hi_to_f32(kw.y), d);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
        const float sc = d * P.sm_scale;
        if (sc == neg_inf()) continue;            // weight 0 against any other score
        const float mn = max_nan(m, sc);          // NaN from the first NaN score on
        const float alpha = __expf(m - mn), p = __expf(sc - mn);
        l = l * alpha + p;
        acc[0] = fmaf(p, bf16lo_to_f32(vw.x), acc[0] * alpha);
        acc[1] = fmaf(p, bf16hi_to_f32(vw.x), acc[1] * alpha);
        acc[2] = fmaf(p, bf16lo_to_f32(vw.y), acc[2] * alpha);
        acc[3] = fmaf(p, bf16hi_to_f32(vw.y), acc[3] * alpha);
        m = mn;
    }
    const bool empty = l == 0.f;                  // nothing visible; a NaN score makes maximum and sum NaN
    const float inv = empty ? 0.f : 1.f / l;
    const float lse = empty ? neg_inf() : m + logf(l);
    if (PREFIX) {
        const size_t o = ((size_t)row * A.out_shards + A.slot) * Hq + h;
        *reinterpret_cast<float4 *>(A.o_part + o * kHeadDim + lane * 4) =
            make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
        if (lane == 0) { A.m_part[o] = m; A.lse_part[o] = lse; }
    } else {
        const size_t o = (size_t)row * Hq + h;
        *reinterpret_cast<uint2 *>(A.out + o * kHeadDim + lane * 4) =
            make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
        if (lane == 0) A.lse[o] = lse;
    }
}

}  // namespace qf
