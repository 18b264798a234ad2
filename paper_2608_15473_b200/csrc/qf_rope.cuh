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
// (offsets, length, table entry).  A CTA walks over steps of a few tokens: eight warps move and turn a step's rows,
// which come through a ring of shared memory (each thread its own words, requested two batches ahead and across steps),
// while a ninth warp looks up the next step's tokens and computes their sines and cosines into the other half of a
// table.  Sixteen lanes own one head row, a 16-byte word each; a word's partner is one shuffle away (or in the word
// itself, interleaved).  The groups of a token take its rows in turn, so that the groups of a warp are always at the
// same kind of row: with consecutive rows per group, warps ran queries, keys and values one after the other at half
// occupancy (15,400 tokens of 32/8 heads with norms: 119 us instead of 81, 4.6 TB/s of 6.5 that a copy reaches).
// Gains and angles meet in one pair of coefficients per channel, kept in registers over the rows of a kind,
//     y_c = (x_c * (g_c cos) + x_partner * (-+ g_partner sin)) / rms,
// two channels per instruction.
#pragma once

#include <mutex>
#include <stddef.h>

#include "qf_common.cuh"
#include "qf_page_math.cuh"

namespace qf {

constexpr int kRopeThreads = 256;                   // that move rows; one more warp prepares the next tokens
constexpr int kRopeGroup = 16;                      // lanes per head row
constexpr int kRopeGroups = kRopeThreads / kRopeGroup;
constexpr int kRopeMaxTokens = 8;                   // per step
constexpr int kRopeBatch = 2;                       // rows of a group that are worked on together
constexpr int kRopeStages = 3;                      // batches in shared memory: one in use, the others on their way
constexpr int kRopeCtasPerSm = 3;

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
    int tokens_per_cta;               // 1, 2, 4 or 8
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

// Two channels, bf16 in a word <-> fp32 in a register pair.
__device__ __forceinline__ unsigned long long pair_of_bf16(uint32_t w)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(w << 16), "r"(w & 0xffff0000u));
    return r;
}
__device__ __forceinline__ unsigned long long pair_of(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split_pair(unsigned long long v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ unsigned long long mul_pair(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long fma_pair(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long swap_pair(unsigned long long v)
{
    float lo, hi;
    split_pair(v, lo, hi);
    return pair_of(hi, lo);
}

// Place and angles of the tokens t0 .. t0 + tokens - 1, by one warp.
struct __align__(16) RopeStep {
    float2 turn[kRopeMaxTokens][64];     // (cos, sin) of every pair
    long long page[kRopeMaxTokens];      // physical page of the token's position, -1 = none
    int slot[kRopeMaxTokens];            // slot within the page; -1: a token of no request
};
static_assert(alignof(RopeStep) >= 16 && offsetof(RopeStep, turn) % 16 == 0, "two pairs of a turn are read as one float4");
__device__ __forceinline__ void rope_prepare(RopeStep &st, const RopeArgs &A, const DevParams &P, int t0, int tokens)
{
    const int lane = threadIdx.x & 31;
    // lane k looks up token k, then all lanes turn its angle
    int b = -1;
    long long pos = 0, base = 0;
    if (lane < tokens && t0 + lane < A.total_tokens) {
        b = request_of(A.cu, P.batch, t0 + lane);
        if (b >= 0) {
            pos = (long long)max(A.seq_lens[b], 0) + ((long long)(t0 + lane) - A.cu[b]);   // not below 0, whatever the offset
            base = A.pos_base ? A.pos_base[b] : 0;
            long long phys = -1;      // nothing is stored where the position has no page
            if (A.k_cache && (pos >> 4) < P.max_pages_per_req) {
                const long long at = (long long)b * P.max_pages_per_req + (pos >> 4);
                phys = A.block_table ? (long long)A.block_table[at] : at;
                if (phys < 0 || phys >= P.num_pages) phys = -1;
            }
            st.page[lane] = phys;
        }
    }
    if (lane < tokens) st.slot[lane] = b >= 0 ? (int)(pos & 15) : -1;
    const int pairs = A.rotary_dim / 2;
    double f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = lane + 32 * i < pairs ? (double)A.inv_freq[lane + 32 * i] * 0.15915494309189533577 : 0.0;   // / (2 pi)
    for (int k = 0; k < tokens; ++k) {
        const double r = (double)__shfl_sync(0xffffffffu, pos + base, k);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = lane + 32 * i;
            if (j >= pairs) continue;
            const double turn = r * f[i];
            float sn, cs;
            sincospif(2.f * (float)(turn - rint(turn)), &sn, &cs);
            st.turn[k][j] = make_float2(cs * A.rot_scale, sn * A.rot_scale);
        }
    }
}

__device__ __forceinline__ void copy_async_16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <bool INTERLEAVED>
__global__ void __launch_bounds__(kRopeThreads + 32, kRopeCtasPerSm)
rope_append_kernel(const __grid_constant__ RopeArgs A, const __grid_constant__ DevParams P)
{
    __shared__ RopeStep steps[2];
    extern __shared__ __align__(16) uint4 ring[];        // [stage][row of the batch][thread]: a thread's own words
    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, lane = tid & (kRopeGroup - 1), group = tid / kRopeGroup;
    const int tokens = A.tokens_per_cta, stride = (int)gridDim.x * tokens;
    int t0 = (int)blockIdx.x * tokens;
    if (tid >= kRopeThreads) {      // the preparing warp: one step ahead
        rope_prepare(steps[0], A, P, t0, tokens);
        __syncthreads();
        for (int n = 1; t0 < A.total_tokens; ++n, t0 += stride) {
            if (t0 + stride < A.total_tokens) rope_prepare(steps[n & 1], A, P, t0 + stride, tokens);
            __syncthreads();
        }
        return;
    }
    const int per_token = kRopeGroups / tokens;          // groups that share a token
    const int my = group / per_token;                    // this group's token of the step
    const int g = group - my * per_token;                // takes rows g, g + per_token, ... of every kind, so that groups agree

    // this lane's eight channels, whether they turn, and the lane of the group that holds their partners
    const int half_chunks = A.rotary_dim >> 4;           // chunks of eight channels in half the rotated part
    const bool turns = lane < 2 * half_chunks, upper = lane >= half_chunks;
    const int partner = INTERLEAVED || !turns ? lane : upper ? lane - half_chunks : lane + half_chunks;
    const int ch = lane * 8, pch = partner * 8;

    // rows by kind: queries, keys, values.  A group's rows of a kind come in batches; a batch is one kind's.
    const int count[3] = {A.n_q, A.n_k, A.rows - A.n_q - A.n_k};
    const int kind0 = g < A.n_q ? 0 : g < A.n_k ? 1 : g < count[2] ? 2 : 3;
    // the batch to be requested next: token, kind, first row
    int rt = t0 + my, r_kind = kind0, r_row = g, r_stage = 0;
    const uint32_t mine = smem_u32(ring + tid);
    auto request = [&]() {
        if (rt < A.total_tokens && kind0 < 3) {          // rows of padding tokens exist; they are dropped later
            const uint16_t *src = (r_kind == 0 ? A.q + (long long)rt * A.q_stride : r_kind == 1 ? A.k + (long long)rt * A.k_stride
                                                                                                : A.v + (long long)rt * A.v_stride) + ch;
#pragma unroll
            for (int i = 0; i < kRopeBatch; ++i) {
                const int h = r_row + i * per_token;
                if (h < count[r_kind]) copy_async_16(mine + (r_stage * kRopeBatch + i) * kRopeThreads * 16, src + h * kHeadDim);
            }
            r_row += kRopeBatch * per_token;
            while (r_kind < 3 && r_row >= count[r_kind]) { ++r_kind; r_row = g; }
            if (r_kind == 3) { r_kind = kind0; rt += stride; }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++r_stage == kRopeStages) r_stage = 0;
    };
    for (int i = 0; i < kRopeStages - 1; ++i) request();
    __syncthreads();
    const unsigned mates = 0xffffu << (threadIdx.x & 16);
    int stage = 0;
    for (int n = 0; t0 < A.total_tokens; ++n, t0 += stride) {
        const RopeStep &st = steps[n & 1];
        const int t = t0 + my;
        const int slot = t < A.total_tokens ? st.slot[my] : -1;
        const long long phys = slot >= 0 ? st.page[my] : -1;
        // the same for every lane of a group
        for (int kind = kind0; t < A.total_tokens && kind < 3; ++kind) {
            if (g >= count[kind]) continue;
            const uint16_t *gain = kind == 0 ? A.q_gain : kind == 1 ? A.k_gain : nullptr;
            const bool works = slot >= 0 && (gain || (kind < 2 && A.rotary_dim > 0));       // else the rows pass through bit for bit
            uint16_t *packed = slot < 0 ? nullptr : kind == 0 ? A.q_out + (long long)t * A.n_q * kHeadDim
                             : kind == 1 && A.k_out ? A.k_out + (long long)t * A.n_k * kHeadDim : nullptr;
            uint16_t *cache = kind > 0 && phys >= 0 ? (kind == 1 ? A.k_cache : A.v_cache) + kv_row_offset(P, phys, 0, slot) : nullptr;
            const long long head_step = P.kv_nhd ? kHeadDim : kPageElems;
            // coefficients of channels 2 i, 2 i + 1 of this lane's eight: own and partner's
            unsigned long long own[4], other[4];
            if (works) {
                uint4 ga = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), gb = ga;
                if (gain) {
                    ga = *reinterpret_cast<const uint4 *>(gain + ch);
                    gb = *reinterpret_cast<const uint4 *>(gain + pch);
                }
                const uint32_t gw[4] = {ga.x, ga.y, ga.z, ga.w}, pw[4] = {gb.x, gb.y, gb.z, gb.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    own[i] = pair_of_bf16(gw[i]);
                    other[i] = 0ull;
                    if (!turns) continue;
                    if (INTERLEAVED) {      // word i is pair 4 lane + i
                        const float2 x = st.turn[my][lane * 4 + i];
                        other[i] = mul_pair(swap_pair(own[i]), pair_of(-x.y, x.y));
                        own[i] = mul_pair(own[i], pair_of(x.x, x.x));
                    } else {
                        const float4 x = *reinterpret_cast<const float4 *>(&st.turn[my][(upper ? pch : ch) + 2 * i]);   // two pairs
                        other[i] = mul_pair(pair_of_bf16(pw[i]), upper ? pair_of(x.y, x.w) : pair_of(-x.y, -x.w));
                        own[i] = mul_pair(own[i], pair_of(x.x, x.z));
                    }
                }
            }
            for (int base = g; base < count[kind]; base += kRopeBatch * per_token) {
                request();
                asm volatile("cp.async.wait_group %0;" ::"n"(kRopeStages - 1) : "memory");
                uint4 wa[kRopeBatch];
#pragma unroll
                for (int i = 0; i < kRopeBatch; ++i) wa[i] = ring[(stage * kRopeBatch + i) * kRopeThreads + tid];
                if (++stage == kRopeStages) stage = 0;
                if (works) {
                    // stage by stage over the batch, so that its rows' shuffles and roots overlap (rows past the end: whatever)
                    unsigned long long scale[kRopeBatch];
                    if (gain) {
                        float ss[kRopeBatch];
#pragma unroll
                        for (int i = 0; i < kRopeBatch; ++i) {
                            const unsigned long long x0 = pair_of_bf16(wa[i].x), x1 = pair_of_bf16(wa[i].y), x2 = pair_of_bf16(wa[i].z), x3 = pair_of_bf16(wa[i].w);
                            float u0, u1, u2, u3;
                            split_pair(fma_pair(x2, x2, mul_pair(x0, x0)), u0, u1);
                            split_pair(fma_pair(x3, x3, mul_pair(x1, x1)), u2, u3);
                            ss[i] = (u0 + u1) + (u2 + u3);
                        }
#pragma unroll
                        for (int off = 1; off < kRopeGroup; off <<= 1)
#pragma unroll
                            for (int i = 0; i < kRopeBatch; ++i) ss[i] += __shfl_xor_sync(mates, ss[i], off);
#pragma unroll
                        for (int i = 0; i < kRopeBatch; ++i) {
                            const float rs = rsqrtf(fmaf(ss[i], 1.0f / kHeadDim, A.eps));
                            scale[i] = pair_of(rs, rs);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kRopeBatch; ++i) scale[i] = pair_of(1.f, 1.f);
                    }
#pragma unroll
                    for (int i = 0; i < kRopeBatch; ++i) {
                        const uint32_t w[4] = {wa[i].x, wa[i].y, wa[i].z, wa[i].w};
                        uint32_t y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const unsigned long long x = pair_of_bf16(w[e]);
                            const unsigned long long px = INTERLEAVED ? swap_pair(x) : pair_of_bf16(__shfl_sync(mates, w[e], partner, kRopeGroup));
                            const unsigned long long own_part = mul_pair(x, own[e]);
                            // channels that do not turn have no partner: an infinity elsewhere must not reach them
                            float v0, v1;
                            split_pair(mul_pair(turns ? fma_pair(px, other[e], own_part) : own_part, scale[i]), v0, v1);
                            y[e] = pack_bf16(v0, v1);
                        }
                        wa[i] = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                }
#pragma unroll
                for (int i = 0; i < kRopeBatch; ++i) {
                    const int h = base + i * per_token;
                    if (h < count[kind]) {
                        if (packed) *reinterpret_cast<uint4 *>(packed + h * kHeadDim + ch) = wa[i];
                        if (cache) *reinterpret_cast<uint4 *>(cache + h * head_step + ch) = wa[i];
                    }
                }
            }
        }
        __syncthreads();
    }
}

inline cudaError_t launch_rope(const RopeArgs &A, const DevParams &P, unsigned blocks, cudaStream_t st)
{
    constexpr int kSmem = kRopeStages * kRopeBatch * kRopeThreads * (int)sizeof(uint4);
    auto kernel = A.interleaved ? rope_append_kernel<true> : rope_append_kernel<false>;
    {   // per-device kernel attribute, set once under a lock
        static std::mutex mu;
        static bool done[2][64];
        int dev = 0;
        cudaGetDevice(&dev);
        std::lock_guard<std::mutex> lock(mu);
        bool &d = done[A.interleaved ? 1 : 0][dev & 63];
        if (!d) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
            if (e != cudaSuccess) return e;
            d = true;
        }
    }
    return launch_pdl(kernel, dim3(blocks), dim3(kRopeThreads + 32), kSmem, st, A, P);
}

}  // namespace qf
