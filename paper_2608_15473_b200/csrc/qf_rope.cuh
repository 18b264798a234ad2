// Placing packed tokens: the norm of every query and key head, the rotary position, the rotated queries out and
// the keys and values into the paged cache, in one pass over the projections' output.
//
// For a token of request b, the i-th of its packed rows, with pos = seq_lens[b] + i its slot in the cache and
// r = pos + pos_base[b] its rotary position, every head row x of q and k becomes
//     y = x / sqrt(mean x^2 + eps) * g                     (skipped without a gain)
//     (y_a, y_b) -> s (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = r * inv_freq[j]
// over the rotary_dim / 2 pairs j; a pair is (j, j + rotary_dim / 2) or, interleaved, (2j, 2j + 1).  Everything
// is fp32 between the one load and the one rounding to bf16 (half a unit in the last place; rounding after the norm
// and again after the rotation would double that).  The angle is the exception: r * inv_freq reaches 1e6 radians, where an fp32
// product is off by 0.06, so it is formed and reduced to a fraction of a turn in fp64 and only that fraction,
// in [-1/2, 1/2], goes to fp32.
//
// Bound: HBM (every byte is read and written once), and for a decode batch the launch and three dependent loads
// (offsets, length, table entry).  Eight lanes own one head row, sixteen channels each as two 16-byte words, so
// that both members of every pair sit in one lane in either pair layout and the norm is three shuffles; a lane
// turns the same pairs of every row it visits, so a token's sines and cosines are computed once per item and
// kept in registers over the item's rows.
#pragma once

#include "qf_common.cuh"
#include "qf_page_math.cuh"

namespace qf {

constexpr int kRopeThreads = 256;
constexpr int kRopeGroup = 8;                       // lanes per head row
constexpr int kRopeItemsPerCta = kRopeThreads / kRopeGroup;

struct RopeArgs {
    const uint16_t *q, *k, *v;        // rows of a token are *_stride elements apart
    uint16_t *q_out, *k_out;          // packed [T, heads, 128]
    uint16_t *k_cache, *v_cache;
    const int *block_table, *cu, *seq_lens, *pos_base;
    const uint16_t *q_gain, *k_gain;
    const float *inv_freq;
    long long q_stride, k_stride, v_stride;
    int total_tokens, rotary_dim, interleaved;
    int rows;                         // head rows per token that this call touches
    int n_q, n_k;                     // of these, query rows first, then key rows, then value rows
    int rows_per_item, items_per_token;
    float eps, rot_scale;
};

// The request that owns packed token t: the last b with cu[b] <= t, if t < cu[b + 1]; -1 for a token of none.
__device__ __forceinline__ int request_of(const int *__restrict__ cu, int batch, int t)
{
    // a decode batch has one token per request: its own index is the answer, in one round trip
    if (t < batch && cu[t] <= t && t < cu[t + 1]) return t;
    int lo = 0, hi = batch;            // cu[lo] <= t < cu[hi] once inside
    if (t < cu[0] || t >= cu[batch]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void unpack8(const uint4 &w, float (&f)[8])
{
    f[0] = bf16lo_to_f32(w.x); f[1] = bf16hi_to_f32(w.x); f[2] = bf16lo_to_f32(w.y); f[3] = bf16hi_to_f32(w.y);
    f[4] = bf16lo_to_f32(w.z); f[5] = bf16hi_to_f32(w.z); f[6] = bf16lo_to_f32(w.w); f[7] = bf16hi_to_f32(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

__global__ void __launch_bounds__(kRopeThreads)
rope_append_kernel(RopeArgs A, DevParams P)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & (kRopeGroup - 1);
    const long long item = (long long)blockIdx.x * kRopeItemsPerCta + threadIdx.x / kRopeGroup;
    const int t = (int)(item / A.items_per_token);
    const int row0 = (int)(item - (long long)t * A.items_per_token) * A.rows_per_item;
    // lanes of a group stay together; a group without a token still takes part in its warp's shuffles
    const int b = t < A.total_tokens ? request_of(A.cu, P.batch, t) : -1;
    const bool live = b >= 0;
    const long long pos = live ? (long long)max(A.seq_lens[b], 0) + (t - A.cu[b]) : 0;

    // the two 16-byte chunks of a row that this lane owns, and whether its pairs turn
    const int half_chunks = A.rotary_dim >> 4;           // chunks of eight channels in half the rotated part
    const bool turns = lane < half_chunks;
    int ca, cb;
    if (A.interleaved) { ca = 2 * lane; cb = ca + 1; }
    else if (turns)    { ca = lane; cb = lane + half_chunks; }
    else               { ca = 2 * lane; cb = ca + 1; }   // channels past the rotated part: chunks 2 half_chunks ..

    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { cs[e] = 1.f; sn[e] = 0.f; }
    if (live && turns && row0 < A.n_q + A.n_k) {
        const double r = (double)(pos + (A.pos_base ? A.pos_base[b] : 0));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double turn = r * (double)A.inv_freq[lane * 8 + e] * 0.15915494309189533577;   // 1 / (2 pi)
            const float frac = (float)(turn - rint(turn));
            sincospif(2.f * frac, &sn[e], &cs[e]);
            sn[e] *= A.rot_scale;
            cs[e] *= A.rot_scale;
        }
    }

    // where the token's rows go in the cache; -1: no page for the position, nothing is stored
    long long phys = -1;
    if (live && A.k_cache && row0 + A.rows_per_item > A.n_q && (pos >> 4) < P.max_pages_per_req) {
        const long long at = (long long)b * P.max_pages_per_req + (pos >> 4);
        phys = A.block_table ? (long long)A.block_table[at] : at;
        if (phys < 0 || phys >= P.num_pages) phys = -1;
    }

    const int row1 = min(row0 + A.rows_per_item, A.rows);
#pragma unroll 4
    for (int r = row0; r < row0 + A.rows_per_item; ++r) {
        const bool is_q = r < A.n_q, is_k = !is_q && r < A.n_q + A.n_k;
        const int h = is_q ? r : is_k ? r - A.n_q : r - A.n_q - A.n_k;
        const bool on = live && r < row1;
        const uint16_t *src = is_q ? A.q + (long long)t * A.q_stride : is_k ? A.k + (long long)t * A.k_stride
                                                                            : A.v + (long long)t * A.v_stride;
        uint4 wa = make_uint4(0, 0, 0, 0), wb = wa;
        if (on) {
            wa = *reinterpret_cast<const uint4 *>(src + h * kHeadDim + ca * 8);
            wb = *reinterpret_cast<const uint4 *>(src + h * kHeadDim + cb * 8);
        }
        if (is_q || is_k) {                              // the same for every lane of a group
            float a[8], c[8];
            unpack8(wa, a);
            unpack8(wb, c);
            const uint16_t *gain = is_q ? A.q_gain : A.k_gain;
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(a[e], a[e], fmaf(c[e], c[e], ss));
            const unsigned group = 0xffu << (threadIdx.x & 24);
#pragma unroll
            for (int off = 1; off < kRopeGroup; off <<= 1) ss += __shfl_xor_sync(group, ss, off);
            if (gain) {
                const float rs = 1.0f / sqrtf(ss * (1.0f / kHeadDim) + A.eps);
                float ga[8], gb[8];
                unpack8(*reinterpret_cast<const uint4 *>(gain + ca * 8), ga);
                unpack8(*reinterpret_cast<const uint4 *>(gain + cb * 8), gb);
#pragma unroll
                for (int e = 0; e < 8; ++e) { a[e] = a[e] * rs * ga[e]; c[e] = c[e] * rs * gb[e]; }
            }
            if (turns) {
                if (A.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float x = a[e], y = a[e + 1], z = c[e], w = c[e + 1];
                        a[e]     = x * cs[e / 2] - y * sn[e / 2];
                        a[e + 1] = y * cs[e / 2] + x * sn[e / 2];
                        c[e]     = z * cs[4 + e / 2] - w * sn[4 + e / 2];
                        c[e + 1] = w * cs[4 + e / 2] + z * sn[4 + e / 2];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = a[e], y = c[e];
                        a[e] = x * cs[e] - y * sn[e];
                        c[e] = y * cs[e] + x * sn[e];
                    }
                }
            }
            if (gain || turns) {   // neither: the row passes through bit for bit
                wa = pack8(a);
                wb = pack8(c);
            }
        }
        if (!on) continue;
        uint16_t *packed = is_q ? A.q_out + ((long long)t * A.n_q + h) * kHeadDim
                         : (is_k && A.k_out) ? A.k_out + ((long long)t * A.n_k + h) * kHeadDim : nullptr;
        if (packed) {
            *reinterpret_cast<uint4 *>(packed + ca * 8) = wa;
            *reinterpret_cast<uint4 *>(packed + cb * 8) = wb;
        }
        if (!is_q && phys >= 0) {
            uint16_t *dst = (is_k ? A.k_cache : A.v_cache) + kv_row_offset(P, phys, h, (int)(pos & 15));
            *reinterpret_cast<uint4 *>(dst + ca * 8) = wa;
            *reinterpret_cast<uint4 *>(dst + cb * 8) = wb;
        }
    }
}

}  // namespace qf
