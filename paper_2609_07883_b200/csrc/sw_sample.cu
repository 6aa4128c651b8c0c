// The draw of one token a row from logits: temperature, top-k, top-p and min-p, by a given uniform number.
//
// Weights are w = exp((x - max) / temperature).  All three limits keep a front part of the logits in falling order (equal ones by index), so what
// they leave is known by one threshold and a number of elements at it, and nothing is sorted.  The token is the first, by index, up to which the
// kept weights sum to more than u times their total.
//
// A border between tokens, or of top-p, is a sum over all logits: with 128256 about equal ones, sums in fp32 would put every tenth draw on the wrong side.
// Weights are worked out in 64 bits (2^x from a table of 16 powers and a polynomial of degree five, 1e-14 off) and rounded to 2^-44 of the
// largest; their sums are integers, exact in any order, and equal logits have equal weights.
//
// A cluster of 1 to 8 CTAs has a row; each CTA copies an equal stretch to shared memory, so logits are read from memory once.  Then
//   - the row's largest logit, and a cut above which some hundreds of logits lie: a quantile of the threads' largest ones (its median over warps and
//     CTAs).  It only has to be about right;
//   - without top-k and top-p, the sums of the weights of every warp's run of logits; the warp that the draw falls into looks for the token;
//   - with them, the logits above the cut are collected in one CTA (another one for the next row; top-p: and all weights summed).  If the threshold lies among
//     them, that CTA has the rest to itself: it keeps them in registers, finds the threshold by radix, 256 bins a pass with their number of logits and
//     weight, and the token likewise, by index.  The others end;
//   - if it does not (a large k, or weights spread over thousands of tokens), all CTAs search their stretches, and read one another's bins: first those
//     above the cut, then 256 bins of equal width over the rest, then the bin that the threshold lies in.
// Bound by the logits' bytes, by the instructions of a weight where all are needed (19 a logit, nine of them in 64 bits), and for a few rows by the
// chain of two cluster barriers and the passes.
#include <cfloat>
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "sw_mixed.cuh"

namespace sw {
namespace cg = cooperative_groups;

constexpr int kSampleBins = 256, kSampleRanks = 8, kMaxWarps = 32;
constexpr int kBlock = 128;   // logits that a warp takes at once
constexpr int kListed = 144;  // logits collected from a CTA
constexpr uint32_t kLowestKey = 0x00800000u;   // key_of() of the lowest finite number
constexpr int kUnitBits = 44;                  // the largest weight is 2^44 units: sums of up to 2^19 of them fit 63 bits

struct SampleShared {
    union {
        uint2 listed[kSampleRanks][kListed];   // the collecting CTA: logits above the cut, as bits, and their indices
        struct {
            uint32_t count[2][kSampleBins], low[2][kSampleBins], high[2][kSampleBins];   // by the parity of the pass: logits, and units in two halves
            uint64_t weight[kSampleBins];                                                // summed over the cluster
            uint32_t number[kSampleBins];                                                // likewise
        } bins;
        uint64_t block[kMaxWarps];   // units of the blocks that the warps look through
    };
    uint2 mine[kListed];
    double power[16];   // (see Weigh)
    uint64_t rank_total[kSampleRanks], rank_above[kSampleRanks], rank_kept[kSampleRanks], warp_sum[kMaxWarps];
    float rank_top[kSampleRanks], rank_cut[kSampleRanks], warp_top[kMaxWarps], warp_cut[kMaxWarps];
    uint32_t rank_listed[kSampleRanks], warp_word[kMaxWarps];
    struct Found {
        uint64_t above_w, w;   // units of what lies above the bin, and in it
        uint32_t above_n, n;
        int bin;               // -1: the target is not reached
    } found;
    uint32_t edge[2], num_mine;
    alignas(16) unsigned char x[];
};

// Floats as integers of the same order; -0 as 0.  (Of a NaN it may be anything: comparisons of the floats come first.)
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// A logit's weight in units: 2^44 2^((x - max) c / 16) with x c to the nearest integer in the exponent and a table of 16 powers, the rest in a polynomial.
// |x c| < 2^36: of large numbers, a temperature below that at which only the largest has a weight is not taken (below).
struct Weigh {
    double c;             // 16 / ln 2 / temperature
    double shift;         // 1.5 2^52 less the largest logit's c, rounded: a sum with it is rounded to an integer, which its low word holds
    float floor;          // weights below 2^-64 are none
    const double* power;  // 2^(44 + (j - f) / 16), f what was rounded off the largest logit's c
    static constexpr uint64_t kZero = 0x4330000000000000ull;   // bits of 2^52: a sum with it is rounded likewise
    static __device__ __forceinline__ double power_of(double f) {   // 2^(f / 16), |f| <= 1/2, to 4.5e-15
        return fma(fma(fma(fma(fma(1.2715658865126869e-09, f, 1.4676444610409443e-07), f, 1.3550807790817295e-05), f, 0.0009383847924862347), f,
                       0.043321698784995775), f, 1.0000000000000044);
    }
    __device__ __forceinline__ uint64_t bits(float x) const {  // kZero + units
        const double d = (double)fmaxf(x, floor), r = fma(d, c, shift), f = fma(d, c, shift - r);   // (NaN: the floor)
        const int n = __double2loint(r);
        const double q = power_of(f);
        const double s = power[n & 15];
        return (uint64_t)__double_as_longlong(fma(q, __hiloint2double(__double2hiint(s) + (n & ~15) * 0x10000, __double2loint(s)), 4503599627370496.0));
    }
    __device__ __forceinline__ uint64_t operator()(float x) const { return bits(x) - kZero; }
};

// share * total, rounded down or up from the exact product (a share of 24 bits times 63); share in [0, 1).
__device__ __forceinline__ uint64_t share_of(float share, uint64_t total, bool up) {
    const uint32_t bits = __float_as_uint(share), e = bits >> 23;
    const uint64_t mantissa = (bits & 0x7fffffu) | (e ? 0x800000u : 0u);
    const int s = 150 - (int)max(e, 1u);   // share = mantissa 2^-s, s >= 24
    const uint64_t lo = mantissa * total, hi = __umul64hi(mantissa, total);
    uint64_t q = 0;
    bool rest = (lo | hi) != 0;
    if (s < 64) {
        q = hi << (64 - s) | lo >> s;
        rest = lo << (64 - s) != 0;
    } else if (s < 128) {
        q = s == 64 ? hi : hi >> (s - 64);
        rest = lo != 0 || (s > 64 && hi << (128 - s) != 0);
    }
    return q + (up && rest);
}

__device__ __forceinline__ uint64_t warp_sum_u64(uint64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ uint64_t warp_scan_u64(uint64_t v, int lane) {   // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}
// the value of one of the first n lanes that `rank` of theirs lie above
__device__ __forceinline__ float lanes_rank(float v, int n, int rank, int lane) {
    int above = 0;
    for (int j = 0; j < n; ++j) {
        const float o = __shfl_sync(0xffffffffu, v, j);
        above += o > v || (o == v && j < lane);
    }
    const unsigned at = __ballot_sync(0xffffffffu, lane < n && above == rank);
    return __shfl_sync(0xffffffffu, v, __ffs(at) - 1);
}

// Four neighbouring logits in shared memory as fp32.
__device__ __forceinline__ void quad_of(const float* x, float (&v)[4]) {
    const float4 q = *reinterpret_cast<const float4*>(x);
    v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void quad_of(const __nv_bfloat16* x, float (&v)[4]) {
    const uint2 q = *reinterpret_cast<const uint2*>(x);
    v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xffff0000u), v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xffff0000u);
}
__device__ __forceinline__ void quad_of(const __half* x, float (&v)[4]) {
    const uint2 q = *reinterpret_cast<const uint2*>(x);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&q.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&q.y));
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
__device__ __forceinline__ float max4(const float (&v)[4]) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }   // (NaN does not count)
__device__ __forceinline__ void store_logit(float* x, float v) { *x = v; }
__device__ __forceinline__ void store_logit(__nv_bfloat16* x, float v) { *x = __float2bfloat16(v); }
__device__ __forceinline__ void store_logit(__half* x, float v) { *x = __float2half(v); }
__device__ __forceinline__ float load_logit(const float* x) { return *x; }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* x) { return __bfloat162float(*x); }
__device__ __forceinline__ float load_logit(const __half* x) { return __half2float(*x); }

// Logits whose keys lie in [lo, hi], in 256 bins: of 2^shift keys each, or (linear) of equal width from x_lo on.
struct Interval {
    uint32_t lo, hi;
    int shift;
    bool linear;
    float x_lo, per;
    __device__ __forceinline__ int bin(float x, uint32_t key) const {
        return linear ? min(kSampleBins - 1, max(0, (int)((x - x_lo) * per))) : (int)((key - lo) >> shift);
    }
    __device__ __forceinline__ void by_key(uint32_t l, uint32_t h) {
        lo = l, hi = h, linear = false;
        shift = max(0, 24 - __clz(h - l));   // (256 << shift > h - l)
    }
};

// The bin in which what lies above it, from above_n logits and above_w units on, reaches the target.  One warp; number(i) and weight(i) of bin i.
template <class N, class W>
__device__ __forceinline__ SampleShared::Found pick_bin(N number, W weight, uint64_t above_n, uint64_t above_w, bool by_weight, uint64_t target, int lane) {
    // lane l has bins 255 - 8 l down to 248 - 8 l
    uint64_t n = 0, w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        n += number(kSampleBins - 1 - lane * 8 - i);
        w += weight(kSampleBins - 1 - lane * 8 - i);
    }
    const uint64_t n_to = above_n + warp_scan_u64(n, lane), w_to = above_w + warp_scan_u64(w, lane);
    const unsigned reached = __ballot_sync(0xffffffffu, (by_weight ? w_to : n_to) >= target);
    n = n_to - n;
    w = w_to - w;
    SampleShared::Found f;
    f.bin = -1;
    f.n = 0;
    f.w = 0;
    const int last = reached ? __ffs(reached) - 1 : 31;
    if (lane == last) {
        for (int i = 0; i < 8 && f.bin < 0; ++i) {
            const int at = kSampleBins - 1 - lane * 8 - i;
            const uint64_t n1 = number(at), w1 = weight(at);
            if (reached && (by_weight ? w + w1 : n + n1) >= target) {
                f.bin = at;
                f.n = (uint32_t)n1;
                f.w = w1;
            } else {
                n += n1;
                w += w1;
            }
        }
        f.above_n = (uint32_t)n;
        f.above_w = w;
    }
    return f;   // (of lane `last`; the caller keeps that one's)
}

// Threads of a CTA, and CTAs an SM: small ones that work while others load, or large ones where no SM gets a second.
constexpr int kManySampleThreads = 1024, kFewSampleThreads = 256;
template <class T, int kSampleThreads>
__global__ void __launch_bounds__(kSampleThreads, kSampleThreads == kFewSampleThreads ? 3 : 1) sw_sample_kernel(const SampleParams p) {
    constexpr int kSampleWarps = kSampleThreads / 32, kHeld = (kListed * kSampleRanks + kSampleThreads - 1) / kSampleThreads;   // kHeld: of the collected logits
    extern __shared__ __align__(16) unsigned char sample_raw[];
    SampleShared& s = *reinterpret_cast<SampleShared*>(sample_raw);
    T* const x = reinterpret_cast<T*>(s.x);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = (int)blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_launch_dependents();
    grid_dependency_wait();
    auto all_here = [&] {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };

    // ---- the row's logits to shared memory, and its settings ----
    // Position i of the stretch is logit first + i; the row's first logit lies `-first` past a 16-byte boundary in CTA 0.
    constexpr int kN = 16 / sizeof(T);
    const T* logits = static_cast<const T*>(p.logits) + row * p.row_stride;
    const int first = rank * p.stretch - (int)((reinterpret_cast<uintptr_t>(logits) & 15) / sizeof(T));
    for (int v = tid; v < p.stretch / kN; v += kSampleThreads) {
        const int e = first + v * kN;
        if (e >= 0 && e + kN <= p.vocab) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(x + v * kN)), "l"(logits + e) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                if (e + i >= 0 && e + i < p.vocab) x[v * kN + i] = logits[e + i];
                else store_logit(&x[v * kN + i], -INFINITY);
            }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (tid < 16) s.power[tid] = exp2((double)kUnitBits + (double)tid / 16.);
    if (tid == 0) s.num_mine = 0;
    const float temperature = p.temperature ? p.temperature[row] : 1.f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f, uniform = p.uniform[row];
    const double usual_c = 16. * 1.4426950408889634 / (double)temperature;
    const bool greedy = !(temperature > 0.f), by_count = !greedy && top_k > 0 && top_k < p.vocab, by_share = !greedy && top_p < 1.f;
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    const int blocks = p.stretch / kBlock, block0 = blocks * warp / kSampleWarps, block1 = blocks * (warp + 1) / kSampleWarps;   // of this warp

    // ---- the largest logit, and the cut ----
    float top = -INFINITY;
#pragma unroll 4
    for (int b = block0; b < block1; ++b) {
        float v[4];
        quad_of(x + b * kBlock + lane * 4, v);
        top = max3(max3(top, v[0], v[1]), v[2], v[3]);
    }
    if (by_count || by_share) {
        // the warp's 32 tops in falling order
#pragma unroll
        for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
            for (int j = k >> 1; j > 0; j >>= 1) {
                const float o = __shfl_xor_sync(0xffffffffu, top, j);
                top = ((lane & j) == 0) == ((lane & k) == 0) ? fmaxf(top, o) : fminf(top, o);
            }
        // With `want` logits above the cut, a share of 1 - exp(-want / threads) of the threads' tops is.
        const float want = by_count ? fmaxf(256.f, 1.5f * (float)top_k + 64.f) : 512.f;
        const int q = min(31, (int)(32.f * (1.f - __expf(-want / (float)(ranks * kSampleThreads)))));
        const float cut = __shfl_sync(0xffffffffu, top, q);
        if (lane == 0) s.warp_top[warp] = top, s.warp_cut[warp] = cut;
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) s.warp_top[warp] = top;
    }
    __syncthreads();
    if (warp == 0) {
        float t = lane < kSampleWarps ? s.warp_top[lane] : -INFINITY;
        float cut = 0.f;
        if (by_count || by_share) cut = lanes_rank(lane < kSampleWarps ? s.warp_cut[lane] : -INFINITY, kSampleWarps, min(kSampleWarps, blocks) / 2, lane);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
        if (lane < ranks) {
            SampleShared* to = cluster.map_shared_rank(&s, lane);
            to->rank_top[rank] = t;
            to->rank_cut[rank] = cut;
        }
    }
    all_here();
    const float rank_top = lane < ranks ? s.rank_top[lane] : -INFINITY;
    float m = rank_top;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = __shfl_sync(0xffffffffu, m, 0);
    if (m == -INFINITY) {   // nothing to draw from
        if (rank == 0 && tid == 0) {
            p.tokens[row] = -1;
            if (p.log_probs) p.log_probs[row] = -INFINITY;
        }
        return;
    }
    if (greedy) {   // the first CTA with that logit has the token
        if (__ffs(__ballot_sync(0xffffffffu, rank_top == m)) - 1 != rank) return;
        uint32_t at = 0xffffffffu;
        for (int b = block0; b < block1; ++b) {
            float v[4];
            quad_of(x + b * kBlock + lane * 4, v);
#pragma unroll
            for (int i = 3; i >= 0; --i)
                if (v[i] == m) at = min(at, (uint32_t)(first + b * kBlock + lane * 4 + i));
        }
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) s.warp_word[warp] = at;
        __syncthreads();
        if (warp == 0) {
            at = __reduce_min_sync(0xffffffffu, lane < kSampleWarps ? s.warp_word[lane] : 0xffffffffu);
            if (lane == 0) {
                p.tokens[row] = (int32_t)at;
                if (p.log_probs) p.log_probs[row] = 0.f;
            }
        }
        return;
    }
    float cut = 0.f;
    if (by_count || by_share) cut = lanes_rank(lane < ranks ? s.rank_cut[lane] : -INFINITY, ranks, ranks / 2, lane);
    if (m == INFINITY) {   // the infinite ones share the draw
        for (int i = tid; i < p.stretch; i += kSampleThreads) store_logit(&x[i], load_logit(&x[i]) == INFINITY ? 0.f : -INFINITY);
        m = cut = 0.f;
        __syncthreads();
    }

    // Temperatures at which no number but the largest logit has a weight are all alike: the next one lies 2^-24 of it below at least, and here 128 times the
    // temperature.
    const uint32_t m_key = key_of(m);
    const float below = fmaxf(value_of(m_key - 1), -FLT_MAX), t = fmaxf(temperature, fabsf(m) * 0x1p-31f);
    Weigh weigh;
    weigh.c = t == temperature ? usual_c : 16. * 1.4426950408889634 / (double)t;
    const double top_c = rint((double)m * weigh.c);
    weigh.shift = 6755399441055744.0 - top_c;
    if (tid < 16) s.power[tid] *= Weigh::power_of(top_c - (double)m * weigh.c);
    weigh.floor = fmaxf(fminf(below, m - 44.3614f * t), -FLT_MAX);   // 64 ln 2
    weigh.power = s.power;
    __syncthreads();
    const bool low = weigh.floor == -FLT_MAX;   // then minus infinity and NaN have to be told from the floor
    const uint64_t least = min_p > 0.f ? (uint64_t)ceil((double)fminf(min_p, 1.f) * (double)weigh(m)) : 0;
    auto block_sum = [&](uint64_t v) {   // (a barrier before the next one)
        v = warp_sum_u64(v);
        if (lane == 0) s.warp_sum[warp] = v;
        __syncthreads();
        return warp_sum_u64(lane < kSampleWarps ? s.warp_sum[lane] : 0);
    };
    // the units of the warp's run of logits, this lane's part
    auto all_units = [&] {
        uint64_t sum = 0;
#pragma unroll 2
        for (int b = block0; b < block1; ++b) {
            float v[4];
            quad_of(x + b * kBlock + lane * 4, v);
            uint64_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = weigh.bits(v[i]);
            if (low) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = v[i] > -INFINITY ? w[i] : Weigh::kZero;
            }
            sum += (w[0] + w[1]) + (w[2] + w[3]);
        }
        return sum - (uint64_t)(4 * (block1 - block0)) * Weigh::kZero;
    };
    auto add_to_bin = [&](int buf, int at, uint64_t u) {
        atomicAdd(&s.bins.count[buf][at], 1u);
        const uint32_t lo = (uint32_t)u, old = atomicAdd(&s.bins.low[buf][at], lo), hi = (uint32_t)(u >> 32) + (old + lo < old);
        if (hi) atomicAdd(&s.bins.high[buf][at], hi);
    };
    auto emit = [&](int token, uint64_t units, uint64_t total) {
        p.tokens[row] = token;
        if (p.log_probs) p.log_probs[row] = (float)log((double)units / (double)total);
    };
    // The draw from weights of `total` units: the token's sum exceeds it.
    auto draw_of = [&](uint64_t total) {
        const float u = fmaxf(uniform, 0.f);
        return u < 1.f ? share_of(u, total, false) : total - 1;
    };

    uint32_t keep = kLowestKey, tie_key = 0, ties = 0, tie_before = 0;   // kept: keys from `keep` on, and the first `ties` logits of the key in front of it
    uint64_t all = 0;
    if (by_count || by_share) {
        // ---- the logits above the cut, collected in one CTA ----
        uint64_t total = by_share && !by_count ? all_units() : 0, above = 0;
#pragma unroll 2
        for (int b = block0; b < block1; ++b) {
            float v[4];
            quad_of(x + b * kBlock + lane * 4, v);
            if (!(max4(v) >= cut)) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] >= cut && v[i] > -INFINITY) {
                    const uint32_t at = atomicAdd(&s.num_mine, 1u);
                    if (at < kListed) s.mine[at] = make_uint2(__float_as_uint(v[i]), (uint32_t)(first + b * kBlock + lane * 4 + i));
                    if (by_share && !by_count) above += weigh(v[i]);
                }
        }
        if (by_share && !by_count) {
            total = block_sum(total);
            __syncthreads();
            above = block_sum(above);
        } else {
            __syncthreads();
        }
        const int collector = row % ranks;
        const uint32_t listed = s.num_mine;
        SampleShared* to = cluster.map_shared_rank(&s, collector);
        if (tid < min(listed, (uint32_t)kListed)) to->listed[rank][tid] = s.mine[tid];
        if (warp == 0 && lane < ranks) {
            SampleShared* peer = cluster.map_shared_rank(&s, lane);
            peer->rank_listed[rank] = listed;
            peer->rank_total[rank] = total;
            peer->rank_above[rank] = above;
        }
        all_here();
        uint32_t n = 0, most = 0;
        above = 0;
        for (int r = 0; r < ranks; ++r) {
            n += s.rank_listed[r];
            most = max(most, s.rank_listed[r]);
            all += s.rank_total[r];
            above += s.rank_above[r];
        }
        uint64_t target = by_count ? (uint64_t)top_k : max((uint64_t)1, share_of(fmaxf(top_p, 0.f), all, true));
        if (most <= kListed && (by_count ? n : above) >= target) {
            if (rank != collector) return;
            uint32_t key[kHeld], order[kHeld];   // order: falls with the index
            uint64_t units[kHeld];
            unsigned live = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                const int at = tid + i * kSampleThreads, r = at / kListed;
                key[i] = order[i] = 0;
                units[i] = 0;
                if (r < ranks && at - r * kListed < (int)s.rank_listed[r]) {
                    const uint2 e = s.listed[r][at - r * kListed];
                    key[i] = key_of(__uint_as_float(e.x));
                    order[i] = ~e.y;
                    units[i] = weigh(__uint_as_float(e.x));
                    live |= 1u << i;
                }
            }
            // Of the held logits in `of`, by falling `k`: leaves in `of` those in front of and in the bin where the target is reached, and in f what
            // that bin is; it has one logit, or one k, or (by number) it is kept whole.
            auto descend = [&](const uint32_t (&k)[kHeld], unsigned& of, uint32_t lo, uint32_t hi, bool by_weight, uint64_t target, uint32_t& bin_lo,
                               uint32_t& bin_hi) {
                uint64_t above_n = 0, above_w = 0;
                for (;;) {
                    const int shift = max(0, 24 - __clz(hi - lo));
                    __syncthreads();
                    if (tid < kSampleBins) s.bins.count[0][tid] = s.bins.low[0][tid] = s.bins.high[0][tid] = 0;
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < kHeld; ++i)
                        if (of >> i & 1 && k[i] >= lo && k[i] <= hi) add_to_bin(0, (int)((k[i] - lo) >> shift), units[i]);
                    __syncthreads();
                    if (warp == 0) {
                        const auto f = pick_bin([&](int i) { return s.bins.count[0][i]; },
                                                [&](int i) { return ((uint64_t)s.bins.high[0][i] << 32) + s.bins.low[0][i]; }, above_n, above_w, by_weight, target, lane);
                        if (f.bin >= 0) s.found = f;
                    }
                    __syncthreads();
                    const auto f = s.found;
                    above_n = f.above_n;
                    above_w = f.above_w;
                    const uint32_t bin_at = lo + ((uint32_t)f.bin << shift);
                    hi = bin_at + min(hi - bin_at, (1u << shift) - 1);
                    lo = bin_at;
                    if (lo == hi || f.n == 1 || (!by_weight && above_n + f.n == target)) {
#pragma unroll
                        for (int i = 0; i < kHeld; ++i)
                            if (k[i] < lo) of &= ~(1u << i);
                        bin_lo = lo;
                        bin_hi = hi;
                        return f;
                    }
                }
            };
            // Keeps the front part of the live logits that reaches the target; of equal ones the first.
            auto cut_to = [&](bool by_weight, uint64_t target) {
                uint32_t lo, hi;
                const auto f = descend(key, live, min(key_of(cut), m_key), m_key, by_weight, target, lo, hi);
                const uint32_t n = by_weight ? (f.w == 0 ? f.n : (uint32_t)min((uint64_t)f.n, (target - f.above_w + f.w / f.n - 1) / (f.w / f.n)))
                                             : (uint32_t)(target - f.above_n);
                if (n == f.n) return;
                unsigned equal = 0;   // (all of one key)
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (live >> i & 1 && key[i] == lo) equal |= 1u << i;
                live &= ~equal;
                descend(order, equal, ~(uint32_t)(p.vocab - 1), ~0u, false, n, lo, hi);
                live |= equal;
            };
            auto live_units = [&] {
                uint64_t sum = 0;
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (live >> i & 1) sum += units[i];
                __syncthreads();
                return block_sum(sum);
            };
            if (by_count) {
                if (n > (uint32_t)top_k) cut_to(false, target);
                if (by_share) target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), live_units(), true));
            }
            if (by_share) cut_to(true, target);
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (units[i] < least) live &= ~(1u << i);
            const uint64_t kept = live_units();
            uint32_t lo, hi;
            unsigned up_to = live;
            descend(order, up_to, ~(uint32_t)(p.vocab - 1), ~0u, true, draw_of(kept) + 1, lo, hi);
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (live >> i & 1 && order[i] >= lo && order[i] <= hi) emit((int)~order[i], units[i], kept);
            return;
        }

        // ---- the threshold lies lower: the lowest key that is kept whole, and how many logits of the key in front of it, by all CTAs ----
        for (int i = tid; i < 2 * kSampleBins; i += kSampleThreads) (&s.bins.count[0][0])[i] = (&s.bins.low[0][0])[i] = (&s.bins.high[0][0])[i] = 0;
        __syncthreads();
        int pass = 0;
        // One pass: bins of the interval's logits, summed over the cluster; then the bin in which what lies above reaches the target.
        auto find = [&](const Interval& iv, uint64_t above_n, uint64_t above_w, bool by_weight, uint64_t target) {
            const int buf = pass & 1;
            if (pass >= 2) {   // (its bins of two passes ago have been read: a barrier lies between)
                if (tid < kSampleBins) s.bins.count[buf][tid] = s.bins.low[buf][tid] = s.bins.high[buf][tid] = 0;
                __syncthreads();
            }
            ++pass;
            const float from = value_of(iv.lo);
            for (int b = block0; b < block1; ++b) {
                float v[4];
                quad_of(x + b * kBlock + lane * 4, v);
                if (!(max4(v) >= from)) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t key = key_of(v[i]);
                    if (v[i] >= from && key >= iv.lo && key <= iv.hi) add_to_bin(buf, iv.bin(v[i], key), weigh(v[i]));
                }
            }
            all_here();
            if (tid < kSampleBins) {
                uint32_t n = 0;
                uint64_t w = 0;
                for (int r = 0; r < ranks; ++r) {
                    const SampleShared* from = cluster.map_shared_rank(&s, r);
                    n += from->bins.count[buf][tid];
                    w += ((uint64_t)from->bins.high[buf][tid] << 32) + from->bins.low[buf][tid];
                }
                s.bins.number[tid] = n;
                s.bins.weight[tid] = w;
            }
            __syncthreads();
            if (warp == 0) {
                const auto f = pick_bin([&](int i) { return s.bins.number[i]; }, [&](int i) { return s.bins.weight[i]; }, above_n, above_w, by_weight, target, lane);
                const unsigned has = __ballot_sync(0xffffffffu, f.bin >= 0);
                if (lane == (has ? __ffs(has) - 1 : 31)) s.found = f;
            }
            __syncthreads();
            return s.found;
        };
        // Keeps the front part that reaches `target` logits, or units, of those from key `bottom` on.
        // Returns the units of what lies above the ties, or is kept whole.
        auto select = [&](Interval iv, uint32_t bottom, bool by_weight, uint64_t target) {
            uint64_t above_n = 0, above_w = 0;
            const uint32_t old_ties = ties;
            for (;;) {
                const auto f = find(iv, above_n, above_w, by_weight, target);
                above_n = f.above_n;
                above_w = f.above_w;
                if (f.bin < 0) {
                    if (iv.lo <= bottom) {   // everything from there on, and of what was kept of the key in front of it
                        keep = bottom;
                        if (by_weight && old_ties > 0) {
                            const uint64_t w = max((uint64_t)1, weigh(value_of(tie_key)));
                            ties = (uint32_t)min((uint64_t)old_ties, target <= above_w ? 0 : (target - above_w + w - 1) / w);
                        }
                        break;
                    }
                    iv.hi = iv.lo - 1;
                    iv.lo = bottom;
                    iv.linear = true;
                    iv.x_lo = fmaxf(weigh.floor, value_of(bottom));
                    iv.per = 256.f / fmaxf(value_of(iv.hi) - iv.x_lo, 1e-30f);
                    continue;
                }
                if (!iv.linear && iv.shift == 0) {   // one key, of equal weights
                    const uint32_t key = iv.lo + f.bin;
                    const uint64_t w = max((uint64_t)1, f.w / f.n);
                    const uint32_t n = (uint32_t)(by_weight ? min((uint64_t)f.n, f.w == 0 ? f.n : (target - above_w + w - 1) / w) : target - above_n);
                    tie_key = key;
                    ties = n == f.n ? 0 : n;
                    tie_before = 0;
                    for (int r = 0; r < rank; ++r) tie_before += cluster.map_shared_rank(&s, r)->bins.count[(pass - 1) & 1][f.bin];
                    keep = n == f.n ? key : key + 1;
                    above_w += n == f.n ? f.w : 0;
                    break;
                }
                uint32_t lo = iv.lo + (iv.linear ? 0 : (uint32_t)f.bin << iv.shift), hi = lo + min(iv.hi - lo, (1u << iv.shift) - 1);
                if (iv.linear) {
                    // the lowest keys of the bin and of the next one: the bin of a number never falls
                    if (tid < 2) {
                        uint32_t a = iv.lo, b = iv.hi + 1;   // (b: past the last)
                        while (a < b) {
                            const uint32_t mid = a + (b - a) / 2;
                            if (iv.bin(value_of(mid), mid) >= f.bin + tid) b = mid;
                            else a = mid + 1;
                        }
                        s.edge[tid] = a;
                    }
                    __syncthreads();
                    lo = s.edge[0];
                    hi = s.edge[1] - 1;
                }
                if (by_weight ? f.n == 1 : above_n + f.n == target) {
                    keep = lo;
                    ties = 0;
                    above_w += f.w;
                    break;
                }
                iv.by_key(lo, hi);
            }
            return above_w;
        };
        Interval iv;
        iv.by_key(max(kLowestKey, key_of(cut)), m_key);
        uint64_t total_k = select(iv, kLowestKey, !by_count, target);
        if (by_count && by_share) {
            if (ties > 0) total_k += ties * weigh(value_of(tie_key));
            target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), total_k, true));
            if (keep <= m_key) {
                iv.by_key(keep, m_key);
                select(iv, keep, true, target);
            } else {   // all of what is left are equal
                const uint64_t w = weigh(value_of(tie_key));
                ties = (uint32_t)min((uint64_t)ties, (target + w - 1) / w);
            }
        }
    }

    // ---- the kept weights' sums ----
    const float tie = value_of(tie_key);
    uint32_t tie_at = 0;   // ties in front of the warp's next block
    if (ties > 0) {
        uint32_t n = 0;
        for (int b = block0; b < block1; ++b) {
            float v[4];
            quad_of(x + b * kBlock + lane * 4, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) n += v[i] == tie;
        }
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) s.warp_word[warp] = n;
        __syncthreads();
        tie_at = tie_before;
        for (int w = 0; w < warp; ++w) tie_at += s.warp_word[w];
    }
    // No logit below this one is kept: of the threshold, or of min_p (less what the rounding of its place can be off).
    float from = value_of(ties > 0 ? tie_key : keep);
    if (least > 0) from = fmaxf(from, fmaxf(-FLT_MAX, m + t * logf(fminf(min_p, 1.f)) * 1.0001f - 1e-5f * (fabsf(m) + t)));
    const bool everything = keep == kLowestKey && least == 0;
    // units of four neighbouring logits of block b, none where they are not kept; `at`: ties so far, moved on
    auto kept_units = [&](int b, uint32_t& at, uint64_t (&w)[4]) {
        float v[4];
        quad_of(x + b * kBlock + lane * 4, v);
        bool in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i] = v[i] >= from && key_of(v[i]) >= keep;
        if (ties > 0) {
            unsigned of[4], any = 0;
            const unsigned lower = (1u << lane) - 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) any |= of[i] = __ballot_sync(0xffffffffu, v[i] == tie);
            if (any) {
                uint32_t mine = at;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mine += __popc(of[i] & lower);
                    at += __popc(of[i]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (of[i] >> lane & 1) in[i] = mine++ < ties;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = 0;
        if (in[0] || in[1] || in[2] || in[3]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = weigh(v[i]);
                if (!in[i] || w[i] < least) w[i] = 0;
            }
        }
    };
    uint64_t sum = 0;
    if (everything) {
        sum = all_units();
    } else {
        uint32_t at = tie_at;
        for (int b = block0; b < block1; ++b) {
            if (ties == 0) {
                float v[4];
                quad_of(x + b * kBlock + lane * 4, v);
                if (!__any_sync(0xffffffffu, max4(v) >= from)) continue;
            }
            uint64_t w[4];
            kept_units(b, at, w);
            sum += (w[0] + w[1]) + (w[2] + w[3]);
        }
    }
    sum = warp_sum_u64(sum);
    __syncthreads();
    if (lane == 0) s.warp_sum[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        const uint64_t cta = warp_sum_u64(lane < kSampleWarps ? s.warp_sum[lane] : 0);
        if (lane < ranks) cluster.map_shared_rank(&s, lane)->rank_kept[rank] = cta;
    }
    all_here();

    // ---- the draw ----
    uint64_t total = 0, in_front = 0;
    for (int r = 0; r < ranks; ++r) {
        total += s.rank_kept[r];
        if (r < rank) in_front += s.rank_kept[r];
    }
    const uint64_t drawn = draw_of(total);
    if (drawn < in_front || drawn >= in_front + s.rank_kept[rank]) return;
    // The warps look through the run of the one that it falls into, a block each.
    int of = 0;
    for (uint64_t w = s.warp_sum[0]; in_front + w <= drawn; w = s.warp_sum[of]) {
        in_front += w;
        ++of;
    }
    const int run0 = blocks * of / kSampleWarps, run1 = blocks * (of + 1) / kSampleWarps;
    for (int round = run0; round < run1; round += kSampleWarps) {
        const int b = round + warp;
        uint64_t w[4] = {0, 0, 0, 0};
        if (b < run1) {
            uint32_t at = tie_before;
            if (ties > 0) {   // those in front of the block
                uint32_t n = 0;
                for (int c = run0; c < b; ++c) {
                    float v[4];
                    quad_of(x + c * kBlock + lane * 4, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) n += v[i] == tie;
                }
                at += __reduce_add_sync(0xffffffffu, n);
                for (int c = 0; c < of; ++c) at += s.warp_word[c];
            }
            kept_units(b, at, w);
        }
        const uint64_t here = (w[0] + w[1]) + (w[2] + w[3]), up_to = warp_scan_u64(here, lane);
        if (round > run0) __syncthreads();
        if (lane == 31) s.block[warp] = up_to;
        __syncthreads();
        uint64_t before = in_front;
        for (int c = 0; c < warp; ++c) before += s.block[c];
        const uint64_t to = before + up_to;
        if (drawn >= to - here && drawn < to) {   // one lane of one warp
            uint64_t at = to - here;
            int i = 0;
            for (; i < 3; ++i) {
                at += w[i];
                if (at > drawn) break;
            }
            emit(first + b * kBlock + lane * 4 + i, i == 0 ? w[0] : i == 1 ? w[1] : i == 2 ? w[2] : w[3], total);
        }
        for (int c = 0; c < kSampleWarps; ++c) in_front += s.block[c];
    }
}

constexpr int kMaxStretch = (227 * 1024 - (int)sizeof(SampleShared)) / 4 / kBlock * kBlock;
static_assert((int64_t)kMaxStretch * kSampleRanks >= kMaxVocab + 8 + kSampleRanks * kBlock, "the largest vocabulary fits eight CTAs");
static_assert(3 * (sizeof(SampleShared) + 16128 * 4 + 1024) <= 228 * 1024, "three stretches of an eighth of 128256 logits fit an SM");

template <class F>
cudaError_t for_each_sample(F f) {
    for (auto* kernel : {sw_sample_kernel<float, kFewSampleThreads>, sw_sample_kernel<float, kManySampleThreads>, sw_sample_kernel<__nv_bfloat16, kFewSampleThreads>,
                         sw_sample_kernel<__nv_bfloat16, kManySampleThreads>, sw_sample_kernel<__half, kFewSampleThreads>, sw_sample_kernel<__half, kManySampleThreads>})
        if (const cudaError_t e = f(kernel)) return e;
    return cudaSuccess;
}
cudaError_t configure_sample_kernels() {
    return for_each_sample([](auto* kernel) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SampleShared) + kMaxStretch * 4);
    });
}

cudaError_t launch_sample(const SampleParams& params, int dtype, int num_sms, cudaStream_t stream) {
    SampleParams p = params;
    const int size = dtype == SW_DTYPE_F32 ? 4 : 2;
    // CTAs of a row: as many as give each 16384 logits at most (64 KB: three CTAs an SM, one loads while the others work), and more where rows are few.
    const int64_t positions = (int64_t)p.vocab + 16 / size - 1;   // (a row may start anywhere behind a 16-byte boundary)
    int ranks = 1;
    while (ranks < kSampleRanks && (positions > ranks * 16384 || (p.rows * ranks < num_sms && positions > ranks * 2048))) ranks *= 2;
    p.stretch = (int)((positions + ranks * kBlock - 1) / (ranks * kBlock) * kBlock);
    const bool many = p.rows * ranks <= num_sms && p.stretch >= 4 * kManySampleThreads;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * ranks));
    cfg.blockDim = dim3(many ? kManySampleThreads : kFewSampleThreads);
    cfg.dynamicSmemBytes = sizeof(SampleShared) + (size_t)p.stretch * size;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    auto launch = [&](auto* few_kernel, auto* many_kernel) { return cudaLaunchKernelEx(&cfg, many ? many_kernel : few_kernel, p); };
    if (dtype == SW_DTYPE_F32) return launch(sw_sample_kernel<float, kFewSampleThreads>, sw_sample_kernel<float, kManySampleThreads>);
    if (dtype == SW_DTYPE_BF16) return launch(sw_sample_kernel<__nv_bfloat16, kFewSampleThreads>, sw_sample_kernel<__nv_bfloat16, kManySampleThreads>);
    return launch(sw_sample_kernel<__half, kFewSampleThreads>, sw_sample_kernel<__half, kManySampleThreads>);
}

}  // namespace sw
