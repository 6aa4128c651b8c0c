// Decode pages of an 8-bit pool on one warp (kKv8), included by sw_mixed.cuh: queries, products and result of a unit.
#pragma once

namespace sw {

// kKv8: what an 8-bit unit carries beside DecodeState.  Its products take f16 operands, into which e4m3 values convert exactly.
//   Queries: a head's row is scaled by a power of two to below 2^15, so its bf16 elements are f16 numbers (those 2^-31 below the largest and more are
//   rounded); q0, q1 undo that for the lane's two heads.
//   Weights: p 2^15 as f16, which is finer than bf16 down to 2^-29 of the largest weight and loses what is 2^-40 below it.
//   V's scales: O is kept in units of `ref`, the scale of a page so far, which follows the pages' scales upward, and downward where a page's is
//   2^-16 of it or less; in between the ratio goes into the page's weights.  Following takes no instruction beside the online softmax's own
//   correction.  `top`: the largest ref; a scale 2^-80 below it (a block of zeros, say) is not followed, or O might overflow.
template <Option O>
struct Kv8State {};
template <>
struct Kv8State<kKv8> {
    float q0, q1, ref, top;
};
constexpr float kKv8WeightBits = 15.f, kKv8WeightUnit = 0.000030517578125f;   // 2^-15
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t f16x2_of_e4m3(uint32_t pair) {   // of the lower two bytes
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((uint16_t)pair));
    return d;
}
__device__ __forceinline__ float2 f32x2_of_f16x2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
__device__ __forceinline__ uint32_t e4m3x4_of(float a, float b, float c, float d) {   // bytes a, b, c, d from the lowest on
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)hi << 16 | lo;
}
// D(16x8, f32) += A(16x16, f16, row) * B(16x8, f16, col)
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The queries as B fragments of Q^T: the lane holds head lane / 4, of every 16 elements 4 (lane % 4) + {0, 1} and + {2, 3}, the order in which
// 8-bit keys come out of their words.
template <int D>
__device__ __forceinline__ void load_query8(const MixedParams& p, int q_row, int kvh, uint32_t (&qb)[D / 16][2], Kv8State<kKv8>& k8) {
    const int lane = threadIdx.x & 31;
    const uint2* src = reinterpret_cast<const uint2*>(p.q + ((int64_t)q_row * p.Hq + kvh * p.group + (lane >> 2)) * D + (lane & 3) * 4);
    uint32_t top = 0;   // bf16 magnitudes compare like integers
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        const uint2 x = (lane >> 2) < p.group ? src[ks * 4] : make_uint2(0u, 0u);
        qb[ks][0] = x.x;
        qb[ks][1] = x.y;
        top = __vmaxu2(top, __vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu));
    }
    top = max(top & 0xffffu, top >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^(14 - exponent of the largest), between 2^-113 and 2^113
    const int e = min(max((int)(top >> 7) - 127, -99), 126);
    const float f = __int_as_float((14 - e + 127) << 23), inverse = __int_as_float((e - 14 + 127) << 23);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int i = 0; i < 2; ++i)
            qb[ks][i] = pack_f16x2(__uint_as_float(qb[ks][i] << 16) * f, __uint_as_float(qb[ks][i] & 0xffff0000u) * f);
    k8.q0 = __shfl_sync(0xffffffffu, inverse, (lane & 3) * 8);       // lanes of heads 2 (lane % 4) and the next
    k8.q1 = __shfl_sync(0xffffffffu, inverse, (lane & 3) * 8 + 4);
    k8.ref = k8.top = 0.f;
}

// One page (K and V of a head at sK, `valid` keys of it attended) in the transposed form of attend_page; scale: of its K and of its V.
// (Two pages at a time, with one correction of O and one set of shuffles for both: one 8192-token context 14.35 -> 13.97 us, but 128 log-normal ones
// 137.4 -> 139.9.)
template <int D>
__device__ __forceinline__ void attend_page8(const MixedParams& p, uint32_t sK, int valid, const uint32_t (&qb)[D / 16][2], DecodeState<D>& st,
                                             Kv8State<kKv8>& k8, float2 scale) {
    constexpr int KS = D / 16, W = D / 32;  // 16-byte chunks of a key, also 16-column tiles of O; words of an eighth of a row
    const int lane = threadIdx.x & 31;
    // S^T = K Q^T for 16 keys, in two chains.  The two words of a lane are its two keys' bytes 4 (lane % 4) .. + 3 of a 16-byte chunk.
    float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};
    const uint32_t addr = D == 128 ? sK + (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) << 4)
                                   : sK + (lane & 15) * 64 + (((lane >> 4) ^ (lane >> 1 & 3)) << 4);
#pragma unroll
    for (int ks = 0; ks < KS; ks += 2) {
        uint32_t r[4];   // keys 0-7 and 8-15 of one chunk, then of the next
        ldmatrix_x4(addr ^ (ks * 16), r[0], r[1], r[2], r[3]);
        mma_f16_16816(s, f16x2_of_e4m3(r[0]), f16x2_of_e4m3(r[1]), f16x2_of_e4m3(r[0] >> 16), f16x2_of_e4m3(r[1] >> 16), qb[ks][0], qb[ks][1]);
        mma_f16_16816(s2, f16x2_of_e4m3(r[2]), f16x2_of_e4m3(r[3]), f16x2_of_e4m3(r[2] >> 16), f16x2_of_e4m3(r[3] >> 16), qb[ks + 1][0], qb[ks + 1][1]);
    }
    // the lane's keys are lane / 4 and lane / 4 + 8; keys past the context are masked
    const float f0 = scale.x * k8.q0, f1 = scale.x * k8.q1;
    const bool ok0 = (lane >> 2) < valid, ok1 = (lane >> 2) + 8 < valid;
    s[0] = ok0 ? (s[0] + s2[0]) * f0 : -INFINITY;
    s[1] = ok0 ? (s[1] + s2[1]) * f1 : -INFINITY;
    s[2] = ok1 ? (s[2] + s2[2]) * f0 : -INFINITY;
    s[3] = ok1 ? (s[3] + s2[3]) * f1 : -INFINITY;
    float mx0 = fmaxf(s[0], s[2]), mx1 = fmaxf(s[1], s[3]);
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, w));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, w));
    }
    mx0 = fmaxf(st.m0, mx0);
    mx1 = fmaxf(st.m1, mx1);
    float c0 = fast_exp2((st.m0 - mx0) * p.sm_scale_log2), c1 = fast_exp2((st.m1 - mx1) * p.sm_scale_log2);
    st.m0 = mx0;
    st.m1 = mx1;
    const float b0 = mx0 * p.sm_scale_log2 - kKv8WeightBits, b1 = mx1 * p.sm_scale_log2 - kKv8WeightBits;
    s[0] = fast_exp2(fmaf(s[0], p.sm_scale_log2, -b0));
    s[1] = fast_exp2(fmaf(s[1], p.sm_scale_log2, -b1));
    s[2] = fast_exp2(fmaf(s[2], p.sm_scale_log2, -b0));
    s[3] = fast_exp2(fmaf(s[3], p.sm_scale_log2, -b1));
    st.l0 = st.l0 * c0 + (s[0] + s[2]);
    st.l1 = st.l1 * c1 + (s[1] + s[3]);
    if (!(scale.y == k8.ref)) {   // V's scale: see Kv8State; warp-uniform
        const float ratio = scale.y / k8.ref;
        if (scale.y > k8.ref || (ratio < 0x1p-16f && scale.y >= k8.top * 0x1p-80f)) {
            c0 *= k8.ref / scale.y;
            c1 *= k8.ref / scale.y;
            k8.ref = scale.y;
            k8.top = fmaxf(k8.top, scale.y);
        } else {   // (a NaN ends here)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] *= ratio;
        }
    }
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        st.o[i][0] *= c0;
        st.o[i][1] *= c1;
        st.o[i][2] *= c0;
        st.o[i][3] *= c1;
    }
    // P^T [keys][heads] as the B operand: keys along the fragment's registers, so the 8x8 blocks are transposed
    const uint32_t p0 = movmatrix_trans(pack_f16x2(s[0], s[1])), p1 = movmatrix_trans(pack_f16x2(s[2], s[3]));
    // O^T += V^T P^T.  A lane's four keys are 2 (lane % 4) + {0, 1} (+ 8), its columns the (lane / 4)-th eighth of the row: the bytes of two keys
    // in one column make a register of V^T, without a transpose.
    uint32_t w[4][W];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 2 * (lane & 3) + (i & 1) + 8 * (i >> 1), c = lane >> 2;
        const uint32_t v8 = sK + kPageSize * D + row * D;
        if constexpr (D == 128)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3])
                         : "r"(v8 + ((c ^ (row & 7)) << 4)) : "memory");
        else
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[i][0]), "=r"(w[i][1])
                         : "r"(v8 + (((c >> 1) ^ (row >> 1 & 3)) << 4) + (c & 1) * 8) : "memory");
    }
    if (valid < kPageSize) {   // slots past the context hold anything, NaN among it
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (2 * (lane & 3) + (i & 1) + 8 * (i >> 1) >= valid) w[i][j] = 0u;
    }
#pragma unroll
    for (int t = 0; t < KS; ++t) {
        const int j = t >> 1;
        const uint32_t sel = t & 1 ? 0x7362 : 0x5140;   // of two keys' words: byte 0 (2) of both, then byte 1 (3) of both
        const uint32_t lo = __byte_perm(w[0][j], w[1][j], sel), hi = __byte_perm(w[2][j], w[3][j], sel);
        mma_f16_16816(st.o[t], f16x2_of_e4m3(lo), f16x2_of_e4m3(lo >> 16), f16x2_of_e4m3(hi), f16x2_of_e4m3(hi >> 16), p0, p1);
    }
}

// stage_result of 8-bit units: the lane's columns are 2 t + {0, 1} of the row's (lane / 4)-th eighth (l is summed over the lanes already).
template <int D>
__device__ __forceinline__ void stage_result8(uint32_t dst, int g, DecodeState<D>& st, const Kv8State<kKv8>& k8) {
    const int lane = threadIdx.x & 31, h = (lane & 3) * 2;
    const float f = k8.ref * kKv8WeightUnit;
    st.l0 *= kKv8WeightUnit;
    st.l1 *= kKv8WeightUnit;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
        const uint32_t at = dst + (h * D + (((lane >> 2) * (D / 8) + 2 * t) ^ (h * 4))) * 4;
        if (h < g) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(st.o[t][0] * f), "f"(st.o[t][2] * f) : "memory");
        if (h + 1 < g) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at + D * 4), "f"(st.o[t][1] * f), "f"(st.o[t][3] * f) : "memory");
    }
    __syncwarp();
}

}  // namespace sw
