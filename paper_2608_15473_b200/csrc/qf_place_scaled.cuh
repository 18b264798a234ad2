// Placing packed tokens into a scaled cache: what qf_rope.cuh does for a bf16 cache, with keys and values stored as one
// byte per channel and one scale per (page, KV head), separately for keys and values.
//
//   number = code * scale,   code an e4m3 number (magnitudes up to M = 448) or an integer (up to M = 127)
//   scale of a block = the smallest 2^k, k >= -100, with |y| <= M 2^k for every row y the block has been given
//
// A block (the 16 rows of one KV head in one page) fills over many calls.  When a row does not fit, the scale grows
// and the codes that earlier calls left in the block are rounded again, to code * old / new.  The ratio is a power
// of two, so for e4m3 nothing but numbers that fall below its smallest normal one changes at all; integers lose the
// bits that leave at the bottom, half a step of the new scale at most.  A block that is written from its first slot on
// starts afresh.  Powers of two cost e4m3 no precision and integers up to one bit of seven against max / M, and buy that
// exactness, exact expansion to bf16, and scales that can be applied anywhere in a product without another rounding.
// Codes are rounded once, from the fp32 result of norm and rotation (half a step; to bf16 first would add 2^-9).
//
// Who does what: a block must be owned by one place, because its scale follows from all of its new rows.  A CTA takes
// the page runs (rows of one request that fall into one page) that BEGIN within its `tile` packed tokens: at most 31
// rows in all.  It forms sines and cosines for these once, then its warps take units: a query head over all rows,
// or the keys or values of one run and KV head.  A warp holds a unit's 16 rows in registers (sixteen lanes per row, 16
// bytes each), finds the largest magnitude, and turns the rows into codes; keys are turned twice rather than kept in
// fp32, which would halve the warps that fit.  gridDim.y splits the KV heads when there are too few runs to fill the GPU.
//
// Bound: HBM for prompts (256 bytes in per head row, 256 out per query and 128 per key or value), latency for a decode batch.
#pragma once

#include "qf_common.cuh"
#include "qf_page_math.cuh"
#include "qf_rope.cuh"

namespace qf {

constexpr int kPlaceWarps = 8;
constexpr int kPlaceTile = 16;             // packed tokens per CTA, at most
constexpr int kPlaceWindow = kPlaceTile + kPageSize - 1;   // rows of the runs that begin in them
constexpr int kPlaceBatch = kPageSize / 2; // row pairs of a run
constexpr int kMinScaleExponent = -100;

// The scale that keeps magnitudes up to `top` in range; NaN if top is not finite.
template <int KV>
__device__ __forceinline__ float scale_for(float top)
{
    constexpr int kTopExponent = KV == kKvE4m3 ? 8 : 6;                              // M = 1.75 * 2^8, (127 / 64) * 2^6
    constexpr unsigned kTopMantissa = KV == kKvE4m3 ? 0x600000u : 0x7e0000u;
    const unsigned bits = __float_as_uint(top) & 0x7fffffffu;
    if (bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const int k = (int)(bits >> 23) - 127 - kTopExponent + ((bits & 0x7fffffu) > kTopMantissa ? 1 : 0);
    return __uint_as_float((unsigned)(max(k, kMinScaleExponent) + 127) << 23);
}
// What a block's stored scale says about the rows it holds: nothing readable counts as no scale at all.
__device__ __forceinline__ float held_scale(float s)
{
    if (s != s || s == __int_as_float(0x7f800000)) return __uint_as_float(0x7fc00000u);
    return s > 0.f ? s : 0.f;
}
// x / s: a product where s is a power of two (every scale that this kernel forms; a caller's own may be anything)
struct Divider {
    float s, inv;
    bool power;
    __device__ __forceinline__ explicit Divider(float by)
    {
        s = by;
        inv = 1.f / by;
        power = (__float_as_uint(by) & 0x7fffffu) == 0;
    }
    __device__ __forceinline__ float operator()(float x) const { return power ? x * inv : x / s; }
};
// Four numbers within range -> four codes, ties to even.
template <int KV>
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d)
{
    if constexpr (KV == kKvE4m3) {
        uint32_t w;
        asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
            "mov.b32 %0, {lo, hi};\n\t}" : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
        return w;
    } else {
        constexpr float kRound = 12582912.f;      // 1.5 * 2^23: the sum's low byte is the rounded integer
        const uint32_t ab = __byte_perm(__float_as_uint(a + kRound), __float_as_uint(b + kRound), 0x0040);
        const uint32_t cd = __byte_perm(__float_as_uint(c + kRound), __float_as_uint(d + kRound), 0x0040);
        return __byte_perm(ab, cd, 0x5410);
    }
}
template <int KV>
__device__ __forceinline__ void numbers_of(uint32_t w, float (&y)[4])
{
    if constexpr (KV == kKvE4m3) {
        __nv_fp8x4_e4m3 v;
        v.__x = w;
        const float4 f = static_cast<float4>(v);
        y[0] = f.x; y[1] = f.y; y[2] = f.z; y[3] = f.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (float)(int8_t)(w >> (8 * i));
    }
}

// A lane's eight channels of a head row, and how they turn.
struct TurnLane {
    int ch, pch, partner;      // first channel, the partners' first channel, the lane of the sixteen that holds them
    bool turns, upper;
};

// Norm and rotation of one row: `w` this lane's eight channels, `turn` the row's (cos, sin) of every pair.
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_row(const uint4 &w, bool works, const uint16_t *gain, const uint4 &own_gain, const uint4 &partner_gain,
                                         const TurnLane &L, const float2 *turn, float eps, float (&y)[8])
{
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { y[2 * i] = bf16lo_to_f32(ww[i]); y[2 * i + 1] = bf16hi_to_f32(ww[i]); }
    if (!works) return;
    float rs = 1.f;
    if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(y[i], y[i], ss);
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
        rs = rsqrtf(fmaf(ss, 1.0f / kHeadDim, eps));
    }
    const uint32_t gw[4] = {own_gain.x, own_gain.y, own_gain.z, own_gain.w};
    const uint32_t pw[4] = {partner_gain.x, partner_gain.y, partner_gain.z, partner_gain.w};
    float p[8];
    if (!INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t o = __shfl_sync(0xffffffffu, ww[i], L.partner, 16);
            p[2 * i] = bf16lo_to_f32(o);
            p[2 * i + 1] = bf16hi_to_f32(o);
        }
    }
    if (gain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[2 * i] *= bf16lo_to_f32(gw[i]); y[2 * i + 1] *= bf16hi_to_f32(gw[i]);
            if (!INTERLEAVED) { p[2 * i] *= bf16lo_to_f32(pw[i]); p[2 * i + 1] *= bf16hi_to_f32(pw[i]); }
        }
    }
    if (L.turns) {      // channels that do not turn have no partner: an infinity elsewhere must not reach them
        if (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {      // word i is pair 4 lane + i
                const float2 t = turn[L.ch / 2 + i];
                const float a = y[2 * i], b = y[2 * i + 1];
                y[2 * i] = fmaf(-b, t.y, a * t.x);
                y[2 * i + 1] = fmaf(a, t.y, b * t.x);
            }
        } else {
            const float4 *t4 = reinterpret_cast<const float4 *>(turn + (L.upper ? L.pch : L.ch));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 t = t4[i];
                y[2 * i] = fmaf(L.upper ? p[2 * i] : -p[2 * i], t.y, y[2 * i] * t.x);
                y[2 * i + 1] = fmaf(L.upper ? p[2 * i + 1] : -p[2 * i + 1], t.w, y[2 * i + 1] * t.z);
            }
        }
    }
    if (gain) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= rs;
    }
}

__device__ __forceinline__ uint4 bf16_row(const float (&y)[8])
{
    return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

template <int KV, bool INTERLEAVED>
__global__ void __launch_bounds__(kPlaceWarps * 32, 2)
place_scaled_kernel(const __grid_constant__ RopeArgs A, float *__restrict__ k_scale, float *__restrict__ v_scale, int tile,
                    const __grid_constant__ DevParams P)
{
    __shared__ __align__(16) float2 turns[kPlaceWindow][64];      // (cos, sin) of every pair
    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int t0 = (int)blockIdx.x * tile;
    // ---- lane k looks up token t0 + k: its request, place and whether a run begins there
    int b = -1, slot = 0, rows_left = 0;
    long long pos = 0, phys = -1;
    if (t0 + lane < A.total_tokens && lane < tile + kPageSize - 1) {
        b = request_of(A.cu, P.batch, t0 + lane);
        if (b >= 0) {
            const long long i = (long long)(t0 + lane) - A.cu[b];
            pos = (long long)max(A.seq_lens[b], 0) + i;
            slot = (int)(pos & (kPageSize - 1));
            rows_left = min(A.cu[b + 1], A.total_tokens) - (t0 + lane);
            if (A.k_cache && (pos >> 4) < P.max_pages_per_req) {      // nothing is stored where the position has no page
                const long long at = (long long)b * P.max_pages_per_req + (pos >> 4);
                phys = A.block_table ? (long long)A.block_table[at] : at;
                if (phys < 0 || phys >= P.num_pages) phys = -1;
            }
        }
    }
    const bool begins = b >= 0 && (slot == 0 || (long long)(t0 + lane) == A.cu[b]);
    const unsigned starts = __ballot_sync(0xffffffffu, begins);
    const unsigned mine = starts & ((1u << tile) - 1);      // runs of this CTA (tile <= 16)
    if (mine == 0) return;                                  // the same for every warp
    const unsigned upto = starts & ((2u << lane) - 1);      // runs that begin at or before this token
    const bool covered = b >= 0 && upto != 0 && ((mine >> (31 - __clz((int)upto))) & 1);
    const unsigned cover = __ballot_sync(0xffffffffu, covered);
    const int lo = __ffs((int)cover) - 1, hi = 32 - __clz((int)cover);      // rows [lo, hi) of the window, with gaps
    // ---- angles: formed and reduced to a fraction of a turn in fp64 (see qf_rope.cuh)
    const int pairs = A.rotary_dim / 2;
    if (pairs > 0) {
        const long long r0 = pos + (b >= 0 && A.pos_base ? A.pos_base[b] : 0);
        for (int k = lo + warp; k < hi; k += kPlaceWarps) {
            if (!((cover >> k) & 1)) continue;
            const long long row_pos = __shfl_sync(0xffffffffu, r0, k);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = lane + 32 * h;
                if (j >= pairs) continue;
                double r = (double)row_pos;
                if (A.positions) {
                    const int axis = min(max(A.pair_axis[j], 0), A.num_axes - 1);
                    r = (double)A.positions[(long long)axis * A.total_tokens + t0 + k];
                }
                const double turn = r * ((double)A.inv_freq[j] * 0.15915494309189533577);      // / (2 pi)
                float sn, cs;
                sincospif(2.f * (float)(turn - rint(turn)), &sn, &cs);
                turns[k][j] = make_float2(cs * A.rot_scale, sn * A.rot_scale);
            }
        }
    }
    __syncthreads();

    // ---- units
    const int Hkv = P.num_kv_heads, G = P.group, parts = (int)gridDim.y, part = (int)blockIdx.y;
    const int heads = (Hkv - part + parts - 1) / parts;                  // KV heads part, part + parts, ...
    const int n_q = A.n_q ? heads * G : 0, n_kv = A.n_k ? heads : 0, n_runs = __popc(mine);
    const int sides = A.v ? 2 : 1;                                       // keys, and values if they are placed
    const int units = n_q + n_runs * n_kv * sides;
    TurnLane L;
    const int l16 = lane & 15, half = lane >> 4, half_chunks = A.rotary_dim >> 4;
    L.ch = l16 * 8;
    L.turns = l16 < 2 * half_chunks;
    L.upper = l16 >= half_chunks;
    L.partner = INTERLEAVED || !L.turns ? l16 : L.upper ? l16 - half_chunks : l16 + half_chunks;
    L.pch = L.partner * 8;
    for (int u = warp; u < units; u += kPlaceWarps) {
        if (u < n_q) {
            // ---- a query head over the window
            const int h = (part + (u / G) * parts) * G + u % G;
            const bool works = A.q_gain || A.rotary_dim > 0;
            uint4 ga = make_uint4(0u, 0u, 0u, 0u), gb = ga;
            if (A.q_gain) {
                ga = *reinterpret_cast<const uint4 *>(A.q_gain + L.ch);
                gb = *reinterpret_cast<const uint4 *>(A.q_gain + L.pch);
            }
            for (int k0 = lo; k0 < hi; k0 += 2 * kPlaceBatch) {
                uint4 w[kPlaceBatch];
#pragma unroll
                for (int i = 0; i < kPlaceBatch; ++i) {
                    const int k = k0 + 2 * i + half;
                    w[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (k < hi && ((cover >> k) & 1))
                        w[i] = __ldcs(reinterpret_cast<const uint4 *>(A.q + (long long)(t0 + k) * A.q_stride + h * kHeadDim + L.ch));
                }
#pragma unroll
                for (int i = 0; i < kPlaceBatch; ++i) {
                    if (k0 + 2 * i >= hi) break;
                    const int k = k0 + 2 * i + half;
                    float y[8];
                    turn_row<INTERLEAVED>(w[i], works, A.q_gain, ga, gb, L, turns[min(k, kPlaceWindow - 1)], A.eps, y);
                    if (k < hi && ((cover >> k) & 1))
                        *reinterpret_cast<uint4 *>(A.q_out + ((long long)(t0 + k) * A.n_q + h) * kHeadDim + L.ch) = bf16_row(y);
                }
            }
            continue;
        }
        // ---- the keys or values of a run and KV head
        const int v = u - n_q, run = v / (n_kv * sides), rest = v - run * n_kv * sides;
        const bool is_v = rest >= n_kv;
        const int c = part + (is_v ? rest - n_kv : rest) * parts;
        unsigned from = mine;
        for (int i = 0; i < run; ++i) from &= from - 1;
        const int k0 = __ffs((int)from) - 1;
        const int s0 = __shfl_sync(0xffffffffu, slot, k0);
        const int n = min(__shfl_sync(0xffffffffu, rows_left, k0), kPageSize - s0);
        const long long page = __shfl_sync(0xffffffffu, phys, k0);
        const uint16_t *src = (is_v ? A.v + (long long)(t0 + k0) * A.v_stride : A.k + (long long)(t0 + k0) * A.k_stride) + c * kHeadDim + L.ch;
        const long long stride = is_v ? A.v_stride : A.k_stride;
        uint8_t *pool = reinterpret_cast<uint8_t *>(is_v ? A.v_cache : A.k_cache);
        float *scale_at = page < 0 ? nullptr : (is_v ? v_scale : k_scale) + page * Hkv + c;
        float old = 0.f;
        if (s0 > 0 && page >= 0) old = held_scale(*scale_at);
        uint4 w[kPlaceBatch];
#pragma unroll
        for (int i = 0; i < kPlaceBatch; ++i) {
            const int r = 2 * i + half;
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < n) w[i] = __ldcs(reinterpret_cast<const uint4 *>(src + r * stride));
        }
        const uint16_t *gain = is_v ? nullptr : A.k_gain;
        const bool works = !is_v && (gain || A.rotary_dim > 0);
        uint4 ga = make_uint4(0u, 0u, 0u, 0u), gb = ga;
        if (gain) {
            ga = *reinterpret_cast<const uint4 *>(gain + L.ch);
            gb = *reinterpret_cast<const uint4 *>(gain + L.pch);
        }
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kPlaceBatch; ++i) {
            if (2 * i >= n) break;
            const int r = 2 * i + half;
            float y[8];
            turn_row<INTERLEAVED>(w[i], works, gain, ga, gb, L, turns[min(k0 + r, kPlaceWindow - 1)], A.eps, y);
            if (r < n) {
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max_nan(top, fabsf(y[e]));
                if (!is_v && A.k_out)
                    *reinterpret_cast<uint4 *>(A.k_out + ((long long)(t0 + k0 + r) * A.n_k + c) * kHeadDim + L.ch) = bf16_row(y);
            }
        }
        if (page < 0) continue;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float scale = max_nan(old, scale_for<KV>(top));
        const Divider by(scale);
        if (s0 > 0 && scale != old) {      // the rows that earlier calls left in the block (a NaN scale is unequal to itself: harmless)
            const float ratio = by(old);
            for (int r = half; r < s0; r += 2) {
                uint2 *at = reinterpret_cast<uint2 *>(pool + kv_row_offset(P, page, c, r) + L.ch);
                const uint2 codes = *at;
                float y0[4], y1[4];
                numbers_of<KV>(codes.x, y0);
                numbers_of<KV>(codes.y, y1);
                *at = make_uint2(codes_of<KV>(y0[0] * ratio, y0[1] * ratio, y0[2] * ratio, y0[3] * ratio),
                                 codes_of<KV>(y1[0] * ratio, y1[1] * ratio, y1[2] * ratio, y1[3] * ratio));
            }
        }
#pragma unroll
        for (int i = 0; i < kPlaceBatch; ++i) {
            if (2 * i >= n) break;
            const int r = 2 * i + half;
            float y[8];
            turn_row<INTERLEAVED>(w[i], works, gain, ga, gb, L, turns[min(k0 + r, kPlaceWindow - 1)], A.eps, y);
            if (r < n)
                *reinterpret_cast<uint2 *>(pool + kv_row_offset(P, page, c, s0 + r) + L.ch) =
                    make_uint2(codes_of<KV>(by(y[0]), by(y[1]), by(y[2]), by(y[3])), codes_of<KV>(by(y[4]), by(y[5]), by(y[6]), by(y[7])));
        }
        if (lane == 0) *scale_at = scale;
    }
}

// One CTA per decode token; prompts in tiles of 16.  KV heads are split until every SM has several CTAs: at 8 requests of
// one token one CTA per head, 16,000 packed tokens two parts.
template <int KV>
inline cudaError_t launch_place_scaled(const RopeArgs &A, float *k_scale, float *v_scale, const DevParams &P, int sms, cudaStream_t st)
{
    int tile = 1;      // about the rows of a request: a CTA's runs share its angles, a decode batch wants a CTA each
    while (tile < kPlaceTile && (long long)A.total_tokens >= 2ll * tile * P.batch) tile *= 2;
    const long long tiles = ((long long)A.total_tokens + tile - 1) / tile;
    int parts = 1;
    while (parts < P.num_kv_heads && tiles * parts < 8ll * sms) parts *= 2;
    if (parts > P.num_kv_heads) parts = P.num_kv_heads;
    auto kernel = A.interleaved ? place_scaled_kernel<KV, true> : place_scaled_kernel<KV, false>;
    return launch_pdl(kernel, dim3((unsigned)tiles, (unsigned)parts), dim3(kPlaceWarps * 32), 0, st, A, k_scale, v_scale, tile, P);
}

}  // namespace qf
