// The step of the decode sweep over a scaled cache (one byte per number): what qf_page_math.cuh's process_page does for a
// bf16 page, for two pages at a time, which have as many bytes.
//
//   s_i = ks * (q . k_i) / sqrt(d),   W += vs * sum_i e^{s_i} v_i        (k_i, v_i codes; ks, vs the page's scales)
//
// Codes become f16 numbers in registers, exactly (e4m3 by the conversion instruction, integers by placing the byte in
// the mantissa of 1024 and subtracting), and go through m16n8k16 products with fp32 accumulators.  Queries become f16
// too: each head is brought to magnitudes below 2^15 by a power of two first.  f16 steps end at 2^-24, so a channel keeps its eight
// significant bits down to 2^-31 of the head's largest, and is off by 2^-39 of the largest at most below that.
// Both scales stay out of the products: ks multiplies the finished score, and the
// weights are taken relative to the two pages' own maximum, times 2^14, so that hi + lo (two f16 terms) are off by 2^-22
// of a weight or by 2^-39 of the two pages' largest: 22 bits down to 2^-17 of the largest, whatever the pages weigh against the
// others.  Each page's product then enters the accumulators with one factor, vs e^{m_pages - m}, so scales take no bits from the
// weights; but 2^-39 of one page's weight may count where the other's values are very much larger (weights 2^-30 of the
// neighbour's under a scale 2^60 times its: 2^-9 of the result).
//
// Fragments.  K: a lane reads 32 channels of rows g and g + 8 (16-byte words 2t and 2t+1 of the swizzled row: eight
// lanes hit eight different bank groups); the words' channels, taken four at a time, are a k-step (which channel is
// which k is free as long as Q agrees).  V: transposing loads move byte pairs (two channels of a token); one byte
// permutation per register separates them, so row g of a 16-channel tile is channel 2g and row g + 8 channel 2g + 1.
// With at most four heads, Q's columns 4..7 repeat columns 0..3, and P's carry lo beside hi: one product instead of two.
//
// Bound: memory, with issue slots close behind.  Per page (4 KB) 290 warp instructions of all roles in e4m3 and 370 in int8,
// counted over 32 requests of 16,384 tokens with four heads per group, where 6.5 TB/s leave an SM about 680 issue slots for
// it.  Such a batch takes 167 to 181 us in e4m3 (6.4 to 5.9 TB/s) and 174 to 187 in int8 in short runs, 185 to 190 and 198 to 205 for
// seconds on end, with one pool or several; with one page per step, and one thread for all copies, 237 and 253 (short runs).
#pragma once

#include "qf_common.cuh"
#include "qf_page_math.cuh"

namespace qf {

// D = A(16x16, row) * B(16x8, col) + D, f16 inputs, fp32 accumulate.
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same with nothing to add to (zeros as an operand, not as registers to be cleared).
__device__ __forceinline__ void mma_f16_fresh(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// (a0, a1) += (x0, x1) * (f0, f1), one instruction
__device__ __forceinline__ void fma_two(float &a0, float &a1, float x0, float x1, float f0, float f1)
{
    asm("{\n\t.reg .b64 a, x, f;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 x, {%2, %3};\n\tmov.b64 f, {%4, %5};\n\t"
        "fma.rn.f32x2 a, x, f, a;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(a0), "+f"(a1) : "f"(x0), "f"(x1), "f"(f0), "f"(f1));
}
__device__ __forceinline__ void mul_two(float &a0, float &a1, float f0, float f1)
{
    asm("{\n\t.reg .b64 a, f;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 f, {%2, %3};\n\tmul.rn.f32x2 a, a, f;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(a0), "+f"(a1) : "f"(f0), "f"(f1));
}
__device__ __forceinline__ void add_two(float &a0, float &a1, float f)
{
    asm("{\n\t.reg .b64 a, f;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 f, {%2, %2};\n\tadd.rn.f32x2 a, a, f;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(a0), "+f"(a1) : "f"(f));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}
__device__ __forceinline__ void unpack_f16(uint32_t w, float &lo, float &hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b)
{
    uint32_t w;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(w) : "r"(a), "r"(b));
    return w;
}
__device__ __forceinline__ uint4 ld_shared_16(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
// Four codes of a word -> f16 pairs: bytes (0, 1) and (2, 3), or, PAIRED, bytes (0, 2) and (1, 3).
template <int KV, bool PAIRED>
__device__ __forceinline__ void halves_of(uint32_t w, uint32_t &first, uint32_t &second)
{
    if constexpr (KV == kKvE4m3) {
        if (PAIRED) w = __byte_perm(w, 0u, 0x3120);
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(first), "=r"(second) : "r"(w));
    } else {
        const uint32_t u = w ^ 0x80808080u;      // code + 128 as the low mantissa byte of 1024: minus 1152 is exact
        first = sub_f16x2(__byte_perm(u, 0x64646464u, PAIRED ? 0x4240 : 0x4140), 0x64806480u);
        second = sub_f16x2(__byte_perm(u, 0x64646464u, PAIRED ? 0x4341 : 0x4342), 0x64806480u);
    }
}

constexpr float kWeightLog2 = 14.f;      // f16 weights of up to 2^14, with room below

// Q's fragments and the factor that its normalisation left out.  qs: the G heads' rows in shared memory.  Returns the factor
// of this lane's head (lane >> 2).
template <int G>
__device__ __forceinline__ float load_q_scaled(const uint16_t *qs, uint32_t (&qf)[8][2], int lane)
{
    const int t = lane & 3, g = G <= 4 ? (lane >> 2) & 3 : lane >> 2;
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (g < G) x = *reinterpret_cast<const uint4 *>(qs + g * kHeadDim + 32 * t + 8 * i);
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
    uint32_t top = 0;      // the largest finite magnitude: infinities and NaN stay what they are
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t a = w[i] & 0x7fffu, b = (w[i] >> 16) & 0x7fffu;
        top = max(top, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = max(top >> 7, 20u);                                 // biased exponent; smaller heads than 2^-107 stay small
    const float down = __uint_as_float((268u - e) << 23);                  // 2^(14 - (e - 127))
#pragma unroll
    for (int i = 0; i < 16; ++i) qf[i >> 1][i & 1] = pack_f16(bf16lo_to_f32(w[i]) * down, bf16hi_to_f32(w[i]) * down);
    return __uint_as_float((e - 14u) << 23);
}

// Two neighbouring pages (32 tokens): one pass for both halves what the softmax costs beside the exponentials, and one page's
// products fill the other's latencies.
// k_base, v_base: shared-memory addresses of the first page's K and V codes ([16 rows][128 B], 128B-swizzled; the second page
// follows); [tlo, thi) rows of each page inside the shard (none of a page that is skipped, whose scales are 0); qs: factors of the
// scores of heads 2t, 2t+1 in units of log 2; m2, l, acc as in process_page, with acc[i][e], acc[i][2 + e] channels 16 i + 2 g
// and 16 i + 2 g + 1 of head 2t + e (FOLD: of the sum of columns 2t + e and 2t + e + 4).
template <int KV, bool FOLD>
__device__ __forceinline__ void process_pages_scaled(uint32_t k_base, uint32_t v_base, const float (&ks)[2], const float (&vs)[2],
                                                     const int (&tlo)[2], const int (&thi)[2], bool ragged, const uint32_t (&qf)[8][2],
                                                     const float (&qs)[2], float (&m2)[2], float (&l)[2], float (&acc)[8][4], int lane)
{
    const int g = lane >> 2, t = lane & 3;
    if (ragged) {
        // values outside the range must contribute nothing, whatever bits they hold: 0 times a NaN is not 0
#pragma unroll 1
        for (int idx = lane; idx < 2 * kScaledPageBytes / 16; idx += 32) {
            const int row = (idx >> 3) & 15;
            const bool second = idx >> 7;
            if (row < (second ? tlo[1] : tlo[0]) || row >= (second ? thi[1] : thi[0])) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_base + idx * 16), "r"(0) : "memory");
        }
        __syncwarp();
    }
    // ---- S[token, head] = K Q^T: sc[p][0], sc[p][1] token g of page p, heads 2t, 2t+1; sc[p][2], sc[p][3] token g + 8
    float sc[2][4];
    uint32_t vr[2][4][4];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        uint32_t kr[2][8];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 x = ld_shared_16(k_base + p * kScaledPageBytes + (g + 8 * r) * 128 + (((2 * t + j) ^ (g & 7)) << 4));
                kr[r][4 * j] = x.x; kr[r][4 * j + 1] = x.y; kr[r][4 * j + 2] = x.z; kr[r][4 * j + 3] = x.w;
            }
        float odd[4];      // two accumulators: half the dependent chain
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            uint32_t a[4];
            halves_of<KV, false>(kr[0][w], a[0], a[2]);
            halves_of<KV, false>(kr[1][w], a[1], a[3]);
            if (w < 2) mma_f16_fresh(w ? odd : sc[p], a, qf[w][0], qf[w][1]);
            else mma_f16(w & 1 ? odd : sc[p], a, qf[w][0], qf[w][1]);
        }
        const float f0 = qs[0] * ks[p], f1 = qs[1] * ks[p];
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[p][i] = (sc[p][i] + odd[i]) * ((i & 1) ? f1 : f0);
        if (ragged) {
            if (g < tlo[p] || g >= thi[p]) { sc[p][0] = neg_inf(); sc[p][1] = neg_inf(); }
            if (g + 8 < tlo[p] || g + 8 >= thi[p]) { sc[p][2] = neg_inf(); sc[p][3] = neg_inf(); }
        }
    }
    const int vrow = (lane & 7) + ((lane >> 3) & 1) * 8, vsel = lane >> 4;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            ldmatrix_x4_trans(vr[p][i], v_base + p * kScaledPageBytes + vrow * 128 + (((2 * i + vsel) ^ (vrow & 7)) << 4));
    // ---- the pages' own softmax
    float mx0 = fmaxf(fmaxf(sc[0][0], sc[0][2]), fmaxf(sc[1][0], sc[1][2])), mx1 = fmaxf(fmaxf(sc[0][1], sc[0][3]), fmaxf(sc[1][1], sc[1][3]));
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) {
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, off));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, off));
    }
    const float mn0 = fmaxf(m2[0], mx0), mn1 = fmaxf(m2[1], mx1);
    const float ms0 = mn0 == neg_inf() ? 0.f : mn0, ms1 = mn1 == neg_inf() ? 0.f : mn1;      // nothing above -inf: avoid inf - inf
    // Weights are taken against the pages' maximum less 14 (in log 2), the same number in w and be, so its rounding cancels.  Pages with
    // no score above -inf (both skipped, say) have weights 0 against any number: the running one, so that be, which they
    // are multiplied by, is 1 and not an infinity that a running maximum far below 0 would make of it.
    const float mp0 = mx0 == neg_inf() ? ms0 : mx0 - kWeightLog2, mp1 = mx1 == neg_inf() ? ms1 : mx1 - kWeightLog2;
    float w[2][4];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[p][i] = fast_exp2(sc[p][i] - ((i & 1) ? mp1 : mp0));
    const float al0 = fast_exp2(m2[0] - ms0), al1 = fast_exp2(m2[1] - ms1);      // of what came before
    const float be0 = fast_exp2(mp0 - ms0), be1 = fast_exp2(mp1 - ms1);          // of these pages
    m2[0] = mn0; m2[1] = mn1;
    l[0] = fmaf(l[0], al0, ((w[0][0] + w[0][2]) + (w[1][0] + w[1][2])) * be0);      // Z from the unrounded weights
    l[1] = fmaf(l[1], al1, ((w[0][1] + w[0][3]) + (w[1][1] + w[1][3])) * be1);
    if (__any_sync(0xffffffffu, (al0 != 1.f) || (al1 != 1.f))) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            mul_two(acc[i][0], acc[i][1], al0, al1);
            mul_two(acc[i][2], acc[i][3], al0, al1);
        }
    }
    // ---- O^T[d, head] += factor * (V^T P^T), P^T as the B operand, hi and lo
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        uint32_t h0 = pack_f16(w[p][0], w[p][1]), h1 = pack_f16(w[p][2], w[p][3]);
        float r0, r1, r2, r3;
        unpack_f16(h0, r0, r1);
        unpack_f16(h1, r2, r3);
        const uint32_t e0 = pack_f16(w[p][0] - r0, w[p][1] - r1), e1 = pack_f16(w[p][2] - r2, w[p][3] - r3);
        uint32_t bl0 = 0u, bl1 = 0u;
        if (FOLD) {
            if (t >= 2) { h0 = e0; h1 = e1; }      // columns 4..7 repeat the heads of 0..3
        } else {
            bl0 = movmatrix_trans(e0);
            bl1 = movmatrix_trans(e1);
        }
        const uint32_t bh0 = movmatrix_trans(h0), bh1 = movmatrix_trans(h1);
        const float vb0 = be0 * vs[p], vb1 = be1 * vs[p];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[4];
            halves_of<KV, true>(vr[p][i >> 1][2 * (i & 1)], a[0], a[1]);
            halves_of<KV, true>(vr[p][i >> 1][2 * (i & 1) + 1], a[2], a[3]);
            float d[4];
            mma_f16_fresh(d, a, bh0, bh1);
            if (!FOLD) mma_f16(d, a, bl0, bl1);
            fma_two(acc[i][0], acc[i][1], d[0], d[1], vb0, vb1);
            fma_two(acc[i][2], acc[i][3], d[2], d[3], vb0, vb1);
        }
    }
}

// One TMA box of a scaled pool: a page of one KV head, 16 rows of 128 B.
__device__ __forceinline__ void tma_load_page_scaled(uint32_t dst, const CUtensorMap *map, int y, int z, uint32_t bar, unsigned long long policy)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;"
        ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(z), "r"(bar), "l"(policy) : "memory");
}
// Four bytes into shared memory, and the arrival on `bar` once all such copies of this thread have landed.
__device__ __forceinline__ void copy_async_4(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(real ? 4 : 0) : "memory");
}
__device__ __forceinline__ void arrive_after_copies(uint32_t bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

}  // namespace qf
