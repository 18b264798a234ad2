// Placing packed tokens into a scaled cache: what qf_rope.cuh does for a bf16 cache, with keys and values stored as one
// byte per channel and one scale per (page, KV head), separately for keys and values.
//
//   number = code * scale,   code an e4m3 number (magnitudes up to M = 448) or an integer (up to M = 127)
//   scale of a block = the smallest 2^k, k >= -100, with |y| <= M 2^k for every row y the block has been given
//
// A block (the 16 rows of one KV head in one page) fills over many calls.  When a row does not fit, the scale grows
// and the codes that earlier calls left in the block are rounded again, to code * old / new.  The ratio is a power
// of two (of the kernel's own scales), so for e4m3 nothing but numbers that fall below its smallest normal one changes at all: they
// lose 2^-10 of each new scale, 2^-9 of the last one in all with the first rounding.  Integers lose the
// bits that leave at the bottom, half a step of the new scale at most.  A block that is written from its first slot on
// starts afresh.  Powers of two cost e4m3 no precision and integers up to one bit of seven against max / M, and buy that
// exactness, exact expansion to bf16, and scales that can be applied anywhere in a product without another rounding.
// Codes are rounded once, from the fp32 result of norm and rotation (half a step; to bf16 first would add 2^-9).
//
// Who does what: a block's scale follows from all of its new rows, so they meet in one CTA.  A CTA takes the page runs (rows of
// one request that fall into one page) that BEGIN within its `tile` packed tokens, in passes of at most 16 rows.  Sixteen
// lanes own a head row (16 bytes each); a warp has two rows, and turns them for one head after the other with the angles and
// gains in registers: all query heads, or an eighth of them when there is but one token.  For keys and values each warp does
// two heads at a time, the rows' largest magnitudes meet in shared memory, and the rows become codes from the registers they
// were turned in.  gridDim.y splits the KV heads when there are too few
// runs to fill the GPU.
//
// Bound: issue slots and latency at 16 warps per SM for prompts (16,000 tokens, 32/8 heads, norms: 102 us, 3.7 TB/s of the 6.5 that
// a copy reaches; 52 % of the issue slots; three CTAs per SM with fewer registers 110 us), the host's call for a decode batch.
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
// What a block's stored scale says about the rows it holds: itself, and NaN for an infinity.  (Scales below zero come from other
// software only; the rows under them are read like any, so they are kept like any.)
__device__ __forceinline__ float held_scale(float s)
{
    return (__float_as_uint(s) & 0x7fffffffu) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : s;
}
// x / s: a product where s is a power of two (every scale that this kernel forms; a caller's own may be anything, also NaN)
struct Divider {
    float s, inv;
    bool power;
    __device__ __forceinline__ explicit Divider(float by)
    {
        const unsigned bits = __float_as_uint(by);
        s = by;
        power = (bits & 0x807fffffu) == 0 && bits - 0x00800000u < 0x7e800000u - 0x00800000u + 1u;      // 2^-126 .. 2^126
        inv = __uint_as_float(0x7f000000u - bits);                                                     // 2^-k
    }
    __device__ __forceinline__ float operator()(float x) const { return power ? x * inv : x / s; }
};
// Four numbers within range -> four codes, ties to even.  (Integers come with 1.5 * 2^23 added, which has rounded them.)
template <int KV>
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d)
{
    if constexpr (KV == kKvE4m3) {
        uint32_t w;
        asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
            "mov.b32 %0, {lo, hi};\n\t}" : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
        return w;
    } else {
        const uint32_t ab = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040);
        const uint32_t cd = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040);
        return __byte_perm(ab, cd, 0x5410);
    }
}
template <int KV>
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d)
{
    constexpr float kRound = 12582912.f, kTop = 127.f;      // (-128 under a scale below zero would round to 128)
    if constexpr (KV == kKvInt8) return pack_codes<KV>(fminf(a, kTop) + kRound, fminf(b, kTop) + kRound, fminf(c, kTop) + kRound, fminf(d, kTop) + kRound);
    else return pack_codes<KV>(a, b, c, d);
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

// Magnitudes travel as 16 bits, two to a word (keys low, values high): the upper half of the fp32 number, with the last bit set
// where the lower half is not 0.  They order like the magnitudes, NaN above infinity, and a scale asks for no more: whether a
// mantissa is above 1.75 or 127/64, whose lower halves are 0.
__device__ __forceinline__ unsigned half_of(float x)
{
    const unsigned bits = __float_as_uint(x) & 0x7fffffffu;
    return (bits >> 16) | ((bits & 0xffffu) ? 1u : 0u);
}
// The largest of sixteen lanes' pairs.  (By shuffles: a reduction instruction for each half of the warp took longer.)
__device__ __forceinline__ unsigned max_of_row(unsigned x)
{
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) x = __vmaxu2(x, __shfl_xor_sync(0xffffffffu, x, off));
    return x;
}
// A lane's eight channels of a head row, and how they turn.  Sixteen lanes own a row, so a warp works on two rows.
struct TurnLane {
    int ch, pch, partner;      // first channel, the partners' first channel, the lane of the sixteen that holds them
    bool turns, upper;
    uint32_t mask;             // all ones where the lane turns: what has no partner must not be reached by another channel's infinity
};
// Where a row's table keeps (cos, sin) of pair j, so that the sixteen lanes' 16-byte reads are neighbours: four words of a lane's
// eight channels in four planes, or, interleaved, its four pairs in two.
template <bool INTERLEAVED>
__device__ __forceinline__ int turn_place(int j)
{
    return INTERLEAVED ? ((j >> 1) & 1) * 32 + (j >> 2) * 2 + (j & 1) : ((j >> 1) & 3) * 16 + (j >> 3) * 2 + (j & 1);
}
// Gain and angle of a row in one pair of coefficients per channel: y_c = (x_c * own_c + x_partner * other_c) / rms.
struct TurnCoefs { unsigned long long own[4], other[4]; };
template <bool INTERLEAVED>
__device__ __forceinline__ TurnCoefs turn_coefs(const uint16_t *gain, const TurnLane &L, const float2 *turn)
{
    TurnCoefs k;
    uint4 ga = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), gb = ga;      // ones
    if (gain) {
        ga = *reinterpret_cast<const uint4 *>(gain + L.ch);
        gb = *reinterpret_cast<const uint4 *>(gain + L.pch);
    }
    const uint32_t gw[4] = {ga.x, ga.y, ga.z, ga.w}, pw[4] = {gb.x, gb.y, gb.z, gb.w};
    const float4 *t4 = reinterpret_cast<const float4 *>(turn);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k.own[i] = pair_of_bf16(gw[i]);
        k.other[i] = 0ull;
        if (!L.turns) continue;
        if (INTERLEAVED) {      // word i is pair 4 lane + i
            const float4 two = t4[(i >> 1) * 16 + L.ch / 8];
            const float c = (i & 1) ? two.z : two.x, sn = (i & 1) ? two.w : two.y;
            k.other[i] = mul_pair(swap_pair(k.own[i]), pair_of(-sn, sn));
            k.own[i] = mul_pair(k.own[i], pair_of(c, c));
        } else {
            const float4 two = t4[i * 8 + (L.upper ? L.pch : L.ch) / 8];
            k.other[i] = mul_pair(pair_of_bf16(pw[i]), L.upper ? pair_of(two.y, two.w) : pair_of(-two.y, -two.w));
            k.own[i] = mul_pair(k.own[i], pair_of(two.x, two.z));
        }
    }
    return k;
}
// Norm and rotation of N rows (of one token, by sixteen lanes each), step by step over all of them so that their shuffles overlap.
template <bool INTERLEAVED, int N>
__device__ __forceinline__ void turn_rows(const uint4 (&w)[N], bool works, bool norm, const TurnCoefs &k, const TurnLane &L, float eps,
                                          unsigned long long (&y)[N][4])
{
#pragma unroll
    for (int b = 0; b < N; ++b) {
        y[b][0] = pair_of_bf16(w[b].x); y[b][1] = pair_of_bf16(w[b].y); y[b][2] = pair_of_bf16(w[b].z); y[b][3] = pair_of_bf16(w[b].w);
    }
    if (!works) return;
    float rs[N];
    if (norm) {
#pragma unroll
        for (int b = 0; b < N; ++b) {
            float u0, u1, u2, u3;
            split_pair(fma_pair(y[b][2], y[b][2], mul_pair(y[b][0], y[b][0])), u0, u1);
            split_pair(fma_pair(y[b][3], y[b][3], mul_pair(y[b][1], y[b][1])), u2, u3);
            rs[b] = (u0 + u1) + (u2 + u3);
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1)
#pragma unroll
            for (int b = 0; b < N; ++b) rs[b] += __shfl_xor_sync(0xffffffffu, rs[b], off);
#pragma unroll
        for (int b = 0; b < N; ++b) rs[b] = rsqrtf(fmaf(rs[b], 1.0f / kHeadDim, eps));
    }
#pragma unroll
    for (int b = 0; b < N; ++b) {
        const uint32_t ww[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pw = (INTERLEAVED ? ww[i] : __shfl_sync(0xffffffffu, ww[i], L.partner, 16)) & L.mask;
            const unsigned long long px = INTERLEAVED ? swap_pair(pair_of_bf16(pw)) : pair_of_bf16(pw);
            y[b][i] = fma_pair(px, k.other[i], mul_pair(y[b][i], k.own[i]));
            if (norm) y[b][i] = mul_pair(y[b][i], pair_of(rs[b], rs[b]));
        }
    }
}
__device__ __forceinline__ uint4 bf16_row(const unsigned long long (&y)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        split_pair(y[i], lo, hi);
        w[i] = pack_bf16(lo, hi);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The codes of a row's eight channels at `to`.
template <int KV>
__device__ __forceinline__ void store_codes(uint8_t *to, const unsigned long long (&y)[4], const Divider &by)
{
    constexpr float kRound = 12582912.f;      // 1.5 * 2^23: the sum's low byte is the rounded integer
    float v[8];
    if (by.power) {
        const unsigned long long inv = pair_of(by.inv, by.inv);
#pragma unroll
        for (int i = 0; i < 4; ++i)      // (a product with a power of two is exact, so the sum rounds once)
            split_pair(KV == kKvInt8 ? fma_pair(y[i], inv, pair_of(kRound, kRound)) : mul_pair(y[i], inv), v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            split_pair(y[i], v[2 * i], v[2 * i + 1]);
            v[2 * i] /= by.s; v[2 * i + 1] /= by.s;
            if (KV == kKvInt8) { v[2 * i] += kRound; v[2 * i + 1] += kRound; }
        }
    }
    *reinterpret_cast<uint2 *>(to) = make_uint2(pack_codes<KV>(v[0], v[1], v[2], v[3]), pack_codes<KV>(v[4], v[5], v[6], v[7]));
}

template <int KV, bool INTERLEAVED>
__global__ void __launch_bounds__(kPlaceWarps * 32, 2)
place_scaled_kernel(const __grid_constant__ RopeArgs A, const __grid_constant__ RopeAxes X, float *__restrict__ k_scale, float *__restrict__ v_scale, int tile,
                    const __grid_constant__ DevParams P)
{
    constexpr int kQ = 4, kKv = 2;                      // heads that a warp works on at a time, the next ones on their way: of queries, KV heads
    __shared__ __align__(16) float2 turns[kPlaceWarps][2][64];      // (cos, sin) of every pair, of a warp's two tokens
    __shared__ unsigned tops[2][kKv * kPlaceWarps][kPageSize];      // every row's largest magnitudes: [turn][head][row]
    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, l16 = lane & 15, half = lane >> 4;
    const int t0 = (int)blockIdx.x * tile;
    // ---- lane k looks up token t0 + k: its request, place and whether a run begins there
    int b = -1, slot = 0;
    long long pos = 0, phys = -1;
    if (t0 + lane < A.total_tokens && lane < tile + kPageSize - 1) {
        b = request_of(A.cu, P.batch, t0 + lane);
        if (b >= 0) {
            pos = (long long)max(A.seq_lens[b], 0) + ((long long)(t0 + lane) - A.cu[b]);
            slot = (int)(pos & (kPageSize - 1));
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
    const unsigned cover = __ballot_sync(0xffffffffu, b >= 0 && upto != 0 && ((mine >> (31 - __clz((int)upto))) & 1));
    const long long rotary = pos + (b >= 0 && A.pos_base ? A.pos_base[b] : 0);

    const int Hkv = P.num_kv_heads, G = P.group, parts = (int)gridDim.y, part = (int)blockIdx.y;
    const int head0 = (int)((long long)part * Hkv / parts), heads = (int)((long long)(part + 1) * Hkv / parts) - head0;      // this part's KV heads
    const int pairs = A.rotary_dim / 2, half_chunks = A.rotary_dim >> 4;
    TurnLane L;
    L.ch = l16 * 8;
    L.turns = l16 < 2 * half_chunks;
    L.upper = l16 >= half_chunks;
    L.mask = L.turns ? 0xffffffffu : 0u;
    L.partner = INTERLEAVED || !L.turns ? l16 : L.upper ? l16 - half_chunks : l16 + half_chunks;
    L.pch = L.partner * 8;

    // ---- passes of whole runs, at most 16 rows of the window each (nearly always one pass)
    unsigned left = mine;
    int turn_no = 0;
    while (left) {
        const int lo = __ffs((int)left) - 1;
        int hi = lo;
        unsigned runs = 0;
        while (left) {      // the run's rows are covered and contiguous, up to the next run's first
            const int k = __ffs((int)left) - 1;
            const unsigned past = (~cover | (starts & ~(1u << k))) & ~((1u << k) - 1);
            const int end = past ? __ffs((int)past) - 1 : 32;
            if (end - lo > kPageSize) break;
            hi = end;
            runs |= 1u << k;
            left &= left - 1;
        }
        const int n_pairs = (hi - lo + 1) >> 1;
        const int slices = n_pairs > 4 ? 8 : n_pairs > 2 ? 4 : n_pairs;      // a warp has one pair of rows, and its share of the heads
        const int pair = warp & (slices - 1), hg = warp / slices, hgs = kPlaceWarps / slices;
        const int k = lo + 2 * pair + half;
        const bool live = k < hi && ((cover >> k) & 1);
        const int my_k = min(k, 31), t = t0 + k;
        const int my_slot = __shfl_sync(0xffffffffu, slot, my_k);
        const long long page = __shfl_sync(0xffffffffu, phys, my_k);
        const bool leads = live && ((runs >> my_k) & 1);                    // this row is its run's first
        // ---- angles: formed and reduced to a fraction of a turn in fp64 (see qf_rope.cuh)
        __syncwarp();
#pragma unroll 1
        for (int r = 0; r < 2; ++r) {
            const int kk = lo + 2 * pair + r;
            if (kk >= hi || !((cover >> kk) & 1)) continue;
            const long long row_pos = __shfl_sync(0xffffffffu, rotary, kk);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = lane + 32 * h;
                if (j >= pairs) continue;
                double x = (double)row_pos;
                if (X.positions)
                    x = (double)X.positions[(long long)min(max(X.pair_axis[j], 0), X.num_axes - 1) * A.total_tokens + t0 + kk];
                const double turn = x * ((double)A.inv_freq[j] * 0.15915494309189533577);      // / (2 pi)
                float sn, cs;
                sincospif(2.f * (float)(turn - rint(turn)), &sn, &cs);
                turns[warp][r][turn_place<INTERLEAVED>(j)] = make_float2(cs * A.rot_scale, sn * A.rot_scale);
            }
        }
        __syncwarp();
        const float2 *turn = turns[warp][half];
        // ---- queries
        if (A.n_q) {
            const bool works = A.q_gain || A.rotary_dim > 0;
            const TurnCoefs co = turn_coefs<INTERLEAVED>(A.q_gain, L, turn);
            const uint16_t *src = A.q + (long long)t * A.q_stride + head0 * G * kHeadDim + L.ch;
            uint16_t *dst = A.q_out + ((long long)t * A.n_q + head0 * G) * kHeadDim + L.ch;
            uint4 w[kQ], next[kQ];
            auto fetch = [&](int i0, uint4 (&to)[kQ]) {
#pragma unroll
                for (int n = 0; n < kQ; ++n) {
                    const int i = i0 + n * hgs;
                    to[n] = make_uint4(0u, 0u, 0u, 0u);
                    if (live && i < heads * G) to[n] = __ldcs(reinterpret_cast<const uint4 *>(src + i * kHeadDim));
                }
            };
            auto finish = [&](int i0, const uint4 (&from)[kQ]) {
#pragma unroll
                for (int n2 = 0; n2 < kQ; n2 += 2) {
                    const uint4 wb[2] = {from[n2], from[n2 + 1]};
                    unsigned long long y[2][4];
                    turn_rows<INTERLEAVED, 2>(wb, works, A.q_gain != nullptr, co, L, A.eps, y);
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const int i = i0 + (n2 + n) * hgs;
                        if (live && i < heads * G) *reinterpret_cast<uint4 *>(dst + i * kHeadDim) = bf16_row(y[n]);
                    }
                }
            };
            fetch(hg, w);
#pragma unroll 1
            for (int i0 = hg; i0 < heads * G; i0 += 2 * kQ * hgs) {
                fetch(i0 + kQ * hgs, next);
                finish(i0, w);
                if (i0 + kQ * hgs >= heads * G) break;
                fetch(i0 + 2 * kQ * hgs, w);
                finish(i0 + kQ * hgs, next);
            }
        }
        if (!A.n_k) continue;
        // ---- keys and values, a few heads at a time: the rows' largest magnitudes meet in shared memory
        const bool works = A.k_gain || A.rotary_dim > 0;
        const TurnCoefs co = turn_coefs<INTERLEAVED>(A.k_gain, L, turn);
        const int first = 31 - __clz((int)(runs & ((2u << my_k) - 1)));      // where this row's run begins
        const int held = my_slot - (k - first);      // rows of earlier calls in the block: those before the run's first slot
        // row l16 of the pass belongs to this row's run
        const bool same = live && lo + l16 >= first && lo + l16 < hi && (31 - __clz((int)(runs & ((2u << (lo + l16)) - 1)))) == first;
        uint4 kw[kKv], vw[kKv], k_next[kKv], v_next[kKv];
        const uint16_t *k_src = A.k + (long long)t * A.k_stride + head0 * kHeadDim + L.ch, *v_src = A.v + (long long)t * A.v_stride + head0 * kHeadDim + L.ch;
        const size_t row_at = kv_row_offset(P, page < 0 ? 0 : page, head0, my_slot) + L.ch, scale_at = (size_t)(page < 0 ? 0 : page) * Hkv + head0;
        uint8_t *k_row = reinterpret_cast<uint8_t *>(A.k_cache) + row_at, *v_row = reinterpret_cast<uint8_t *>(A.v_cache) + row_at;
        float *ks_at = k_scale + scale_at, *vs_at = v_scale + scale_at;
        const int head_step = P.kv_nhd ? kHeadDim : kPageElems, row_step = P.kv_nhd ? Hkv * kHeadDim : kHeadDim;
        const bool placed = live && page >= 0;
        auto fetch = [&](int c0, uint4 (&to_k)[kKv], uint4 (&to_v)[kKv]) {
#pragma unroll
            for (int n = 0; n < kKv; ++n) {
                const int i = c0 + hg + n * hgs;
                to_k[n] = to_v[n] = make_uint4(0u, 0u, 0u, 0u);
                if (!live || i >= heads) continue;
                to_k[n] = __ldcs(reinterpret_cast<const uint4 *>(k_src + i * kHeadDim));
                if (A.v) to_v[n] = __ldcs(reinterpret_cast<const uint4 *>(v_src + i * kHeadDim));
            }
        };
        fetch(0, kw, vw);
#pragma unroll 1
        for (int c0 = 0; c0 < heads; c0 += kKv * hgs, turn_no ^= 1) {
            fetch(c0 + kKv * hgs, k_next, v_next);
            float old_k[kKv], old_v[kKv];      // the scales that earlier calls left with the block, if they left rows
#pragma unroll
            for (int n = 0; n < kKv; ++n) {
                const int i = c0 + hg + n * hgs;
                old_k[n] = old_v[n] = 0.f;
                if (placed && held > 0 && i < heads) { old_k[n] = __ldcg(ks_at + i); old_v[n] = __ldcg(vs_at + i); }
            }
            unsigned long long y[kKv][4];
            turn_rows<INTERLEAVED, kKv>(kw, works, A.k_gain != nullptr, co, L, A.eps, y);
#pragma unroll
            for (int n = 0; n < kKv; ++n) {
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v0, v1;
                    split_pair(y[n][e], v0, v1);
                    top = max3_nan(top, fabsf(v0), fabsf(v1));
                }
                const uint32_t a = __vmaxu2(__vmaxu2(vw[n].x & 0x7fff7fffu, vw[n].y & 0x7fff7fffu), __vmaxu2(vw[n].z & 0x7fff7fffu, vw[n].w & 0x7fff7fffu));
                const unsigned both = max_of_row(half_of(top) | (__vmaxu2(a, a << 16) & 0xffff0000u));
                if (live && l16 == 0) tops[turn_no][hg * kKv + n][k - lo] = both;
            }
            if (A.k_out && live) {
#pragma unroll
                for (int n = 0; n < kKv; ++n) {
                    const int i = c0 + hg + n * hgs;
                    if (i < heads) *reinterpret_cast<uint4 *>(A.k_out + ((long long)t * A.n_k + head0 + i) * kHeadDim + L.ch) = bf16_row(y[n]);
                }
            }
            __syncthreads();      // (the other half of `tops` is free by now: its readers came before this barrier)
            unsigned top[kKv];
#pragma unroll
            for (int n = 0; n < kKv; ++n) top[n] = max_of_row(same ? tops[turn_no][hg * kKv + n][l16] : 0u);
            const uint4 v_now[kKv] = {vw[0], vw[1]};
#pragma unroll
            for (int n = 0; n < kKv; ++n) { kw[n] = k_next[n]; vw[n] = v_next[n]; }
            if (!placed) continue;
#pragma unroll
            for (int n = 0; n < kKv; ++n) {
                const int i = c0 + hg + n * hgs;
                if (i >= heads) break;
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    const float old = held > 0 ? held_scale(side ? old_v[n] : old_k[n]) : 0.f;
                    const float least = max_nan(fabsf(old), scale_for<KV>(__uint_as_float(side ? top[n] & 0xffff0000u : top[n] << 16)));
                    const float scale = fabsf(old) == least ? old : least;      // the present one where it suffices, with its sign
                    const Divider by(scale);
                    uint8_t *to = (side ? v_row : k_row) + (size_t)i * head_step;
                    if (leads) {
                        if (held > 0 && scale != old) {      // (a NaN scale is unequal to itself: harmless)
                            const float ratio = by(old);
                            for (int r = 1; r <= held; ++r) {
                                uint2 *at = reinterpret_cast<uint2 *>(to - (size_t)r * row_step);
                                const uint2 codes = *at;
                                float y0[4], y1[4];
                                numbers_of<KV>(codes.x, y0);
                                numbers_of<KV>(codes.y, y1);
                                *at = make_uint2(codes_of<KV>(y0[0] * ratio, y0[1] * ratio, y0[2] * ratio, y0[3] * ratio),
                                                 codes_of<KV>(y1[0] * ratio, y1[1] * ratio, y1[2] * ratio, y1[3] * ratio));
                            }
                        }
                        if (l16 == 0) (side ? vs_at : ks_at)[i] = scale;
                    }
                    if (side == 0) {
                        store_codes<KV>(to, y[n], by);
                    } else {
                        const unsigned long long v[4] = {pair_of_bf16(v_now[n].x), pair_of_bf16(v_now[n].y), pair_of_bf16(v_now[n].z), pair_of_bf16(v_now[n].w)};
                        store_codes<KV>(to, v, by);
                    }
                }
            }
        }
    }
}

// One CTA per decode token; prompts in tiles of up to 16.  KV heads are split until every SM has its two CTAs: 8 requests of one
// token take a CTA per head, 16,000 packed tokens one part.
template <int KV>
inline cudaError_t launch_place_scaled(const RopeArgs &A, const RopeAxes &X, float *k_scale, float *v_scale, const DevParams &P, int sms, cudaStream_t st)
{
    int tile = 1;      // about the rows of a request: a CTA's runs share its angles, a decode batch wants a CTA each
    while (tile < kPlaceTile && (long long)A.total_tokens >= 2ll * tile * P.batch) tile *= 2;
    const long long tiles = ((long long)A.total_tokens + tile - 1) / tile;
    int parts = 1;
    while (parts < P.num_kv_heads && tiles * parts < 2ll * sms) parts *= 2;
    if (parts > P.num_kv_heads) parts = P.num_kv_heads;
    auto kernel = A.interleaved ? place_scaled_kernel<KV, true> : place_scaled_kernel<KV, false>;
    return launch_pdl(kernel, dim3((unsigned)tiles, (unsigned)parts), dim3(kPlaceWarps * 32), 0, st, A, X, k_scale, v_scale, tile, P);
}

}  // namespace qf
