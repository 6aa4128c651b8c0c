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
// A cluster of 1 to 8 CTAs has a row, each CTA an equal stretch of it and each warp a run of that.  As much of the runs as there is room for is copied to shared
// memory; the rest is read again where it is needed, from L2.  Then
//   - the row's largest logit, and a cut above which some hundreds of logits lie: a quantile of the threads' largest ones (its median over warps and
//     CTAs).  It only has to be about right;
//   - without top-k and top-p, the sums of the weights of every run; the CTA that the draw falls into looks for the token in one of its runs;
//   - with them, the logits above the cut are collected in one CTA (another one for the next row; top-p: and all weights summed).  If the threshold lies among
//     them, that CTA has the rest to itself: it keeps them in registers, finds the threshold by radix, 256 bins a pass with their number of logits and
//     weight, and the token likewise, by index.  The others end;
//   - if it does not, and there is no top-k (weights spread over thousands of tokens): an eighth of the logits tell about where the threshold lies, the weights
//     above three places around it where it lies to some hundreds of logits, and these are collected, and the threshold found among them, as before;
//   - otherwise (a large k, more than hundreds of equal logits at the threshold) all CTAs search their stretches by bins, and read one another's.
// Bound by the logits' bytes, by the instructions of a weight where all are needed (some 20 a logit, nine of them in 64 bits, and a conversion), and for a
// few rows by the chain of two cluster barriers and the passes.
// Measured, launches in a graph: one row of 128256 fp32 logits 8.5 us, the largest alone 3.9, top-k 50 12.2, with top-p too 13.4, min-p 7.8, 0.95 of an open row 37; 256 such
// rows (131 MB, 20 us at a copy's rate) 71, 29, 64, 68, 64 and 342; 128 rows of 32003 without limits 14.1.  256 rows of 16 bits (10 us of bytes) 71, 27, 64, 69 and 66.
// So bytes bound none of them.  The largest alone: a CTA loads, then compares, then ends, and three an SM overlap that in part (issue slots 37 %).  Top-k: one CTA of the row has the
// searches, a chain of barriers, and its third of the SM's shared memory meanwhile (issue slots 36 %).  Min-p: few weights (64-bit pipes 4 %),
// but a second sweep that looks block by block whether there are any (49 %).  Without limits: the weights take 27 us of the 64-bit pipes and the conversions alone
// (30 cycles for 32 logits and scheduler); the rest of the 71 is loads, sums and the waits for both, as a third CTA an SM hides a part of them only.
// With three CTAs an SM a thread has 80 registers and spills (68 bytes in fp32, 116 and 128 with 16-bit logits); the other kernels, with 120 to
// 128 registers, do not.
#include <cfloat>
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "sw_mixed.cuh"

namespace sw {
namespace cg = cooperative_groups;

constexpr int kSampleBins = 256, kSampleRanks = 8, kMaxWarps = 16;
constexpr int kBlock = 128, kFar = 4;   // logits that a warp takes at once; such blocks outside shared memory that it loads at once
constexpr int kListed = 1024;  // logits that can be collected: an equal part from each CTA
constexpr uint32_t kLowestKey = 0x00800000u;   // key_of() of the lowest finite number
constexpr int kUnitBits = 44;                  // the largest weight is 2^44 units: sums of up to 2^19 of them fit 63 bits

struct SampleShared {
    union {
        uint2 listed[kListed];   // logits above the cut, as bits, and their indices: a part for each CTA, in its own place here and in the collecting CTA
        uint32_t bins[2][4][kSampleBins];   // by the parity of the pass: logits, and units in three parts of 15 bits
        uint64_t block[kMaxWarps];   // units of the blocks that the warps look through
    };
    double power[16];   // (see Weigh)
    uint64_t rank_total[kSampleRanks], rank_above[kSampleRanks], rank_kept[kSampleRanks], warp_sum[kMaxWarps], pick_w[8];
    float rank_top[kSampleRanks], rank_cut[kSampleRanks], warp_top[kMaxWarps], warp_cut[kMaxWarps];
    uint32_t rank_listed[kSampleRanks], warp_word[kMaxWarps], pick_n[8];
    struct Found {
        uint64_t above_w, w;   // units of what lies above the bin, and in it
        uint32_t above_n, n;
        int bin;               // -1: the target is not reached
    } found;
    uint32_t edge[2], num_mine;
    uint32_t front[4];       // from the collecting CTA: keep, and the key in front of it with the last index that is kept of it
    uint64_t rank_places[kSampleRanks][3];
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
// A sum with 2^52, and with such sums up to 2^53, is rounded to an integer: so the weight is added as it is rounded.
struct Weigh {
    double c;             // 16 / ln 2 / temperature
    double shift;         // 1.5 2^52 less the largest logit's c, rounded: a sum with it is rounded to an integer, which its low word holds
    float floor;          // weights below 2^-64 are none
    const double* power;  // 2^(44 + (j - f) / 16), f what was rounded off the largest logit's c; j 2^48 less, as integers
    static constexpr double kZero = 4503599627370496.0;   // 2^52
    static __device__ __forceinline__ double power_of(double f) {   // 2^(f / 16), |f| <= 1/2, to 4.5e-15
        return fma(fma(fma(fma(fma(1.2715658865126869e-09, f, 1.4676444610409443e-07), f, 1.3550807790817295e-05), f, 0.0009383847924862347), f,
                       0.043321698784995775), f, 1.0000000000000044);
    }
    __device__ __forceinline__ void factors(float x, double& a, double& b) const {
        const double d = (double)fmaxf(x, floor), r = fma(d, c, shift), f = fma(d, c, shift - r);   // (NaN: the floor)
        const int n = __double2loint(r);
        const double s = power[n & 15];
        a = power_of(f);
        b = __hiloint2double(__double2hiint(s) + n * 0x10000, __double2loint(s));
    }
    __device__ __forceinline__ double add(float x, double sum) const {   // sum: kZero and units
        double a, b;
        factors(x, a, b);
        return fma(a, b, sum);
    }
    static __device__ __forceinline__ uint64_t units(double sum) { return (uint64_t)(__double_as_longlong(sum) - __double_as_longlong(kZero)); }
    __device__ __forceinline__ uint64_t operator()(float x) const { return units(add(x, kZero)); }
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

// Bits at the end of a key in which the logits of one sign do not differ: so many neighbouring keys hold one logit at most.
template <class T>
constexpr int kGrain = 0;
template <>
constexpr int kGrain<__nv_bfloat16> = 16;
template <>
constexpr int kGrain<__half> = 13;
template <class T>
__device__ __forceinline__ uint32_t only_key(uint32_t lo) {   // the one of keys [lo, lo + 2^kGrain)
    constexpr uint32_t kLow = (1u << kGrain<T>) - 1;
    if (kLow == 0) return lo;
    if (lo < 0x80000000u && (lo | kLow) != 0x7fffffffu) return lo | kLow;   // (keys of negative numbers end in ones; there is no -0)
    return (max(lo, 0x80000000u) + kLow) & ~kLow;
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
    int shift = 0;
    bool linear;
    float x_lo = 0.f, per = 0.f;
    __device__ __forceinline__ int bin(float x, uint32_t key) const {
        return linear ? min(kSampleBins - 1, max(0, (int)((x - x_lo) * per))) : (int)((key - lo) >> shift);
    }
    __device__ __forceinline__ void by_key(uint32_t l, uint32_t h, int grain) {
        lo = l, hi = h, linear = false;
        shift = max(grain, 24 - __clz(h - l));   // (256 << shift > h - l)
    }
    __device__ __forceinline__ void over(uint32_t l, uint32_t h, float floor) {   // what lies below `floor` is in the first bin
        lo = l, hi = h, linear = true;
        x_lo = fmaxf(floor, value_of(l));
        per = (float)kSampleBins / fmaxf(value_of(h) - x_lo, 1e-30f);
    }
};

// (What runs once or twice a row is not inlined: the kernels stay small, and no slower.)
__device__ __noinline__ uint64_t units_once(double c, double shift, float floor, const double* power, float x) { return Weigh{c, shift, floor, power}(x); }

// The bin, from the highest on, in which what lies above, above_n logits and above_w units included, reaches the target.  Thread i < 256 brings the
// n logits and w units of bin 255 - i.
__device__ __noinline__ void pick(SampleShared& s, uint32_t n, uint64_t w, uint32_t above_n, uint64_t above_w, bool by_weight, uint64_t target) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t n_to = n;
    uint64_t w_to = w;
    if (warp < 8) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t a = __shfl_up_sync(0xffffffffu, n_to, o);
            const uint64_t b = __shfl_up_sync(0xffffffffu, w_to, o);
            if (lane >= o) n_to += a, w_to += b;
        }
        if (lane == 31) s.pick_n[warp] = n_to, s.pick_w[warp] = w_to;
    }
    __syncthreads();
    if (warp < 8) {
        n_to += above_n;
        w_to += above_w;
        for (int i = 0; i < warp; ++i) n_to += s.pick_n[i], w_to += s.pick_w[i];
        const uint64_t to = by_weight ? w_to : n_to, before = by_weight ? w_to - w : n_to - n;
        if (before < target && (to >= target || tid == kSampleBins - 1)) {
            const bool here = to >= target;
            s.found.bin = here ? kSampleBins - 1 - tid : -1;
            s.found.n = here ? n : 0;
            s.found.w = here ? w : 0;
            s.found.above_n = here ? n_to - n : n_to;
            s.found.above_w = here ? w_to - w : w_to;
        }
    }
    __syncthreads();
}

// kCtas: CTAs an SM, of 256 threads, so that some work while others load, or of 512 where no SM gets a second one.  (Three of 384, or two of 512, which have
// fewer registers a thread or a barrier for more warps: 256 rows of 128256 without limits 82 and 88 us instead of 70; where two an SM are all there are, 80
// registers a thread instead of 128 make 128 rows of 32003 18.1 us instead of 14.1; 1024 threads one row of 128256 10.5 instead of 8.4.)
template <int kCtas>
constexpr int kThreadsFor = kCtas == 1 ? 512 : 256;
template <class T, int kCtas>
__global__ void __launch_bounds__(kThreadsFor<kCtas>, kCtas) sw_sample_kernel(const SampleParams p) {
    constexpr int kSampleThreads = kThreadsFor<kCtas>;
    constexpr int kSampleWarps = kSampleThreads / 32, kHeld = kListed / kSampleThreads;   // kHeld: of the collected logits
    extern __shared__ __align__(16) unsigned char sample_raw[];
    SampleShared& s = *reinterpret_cast<SampleShared*>(sample_raw);
    T* const x = reinterpret_cast<T*>(s.x);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = (int)blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (ranks > 1) cluster_arrive();   // (waited for in front of the first store to another CTA, behind the loads)
    grid_launch_dependents();
    grid_dependency_wait();
    auto all_here = [&] {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };

    // ---- the row's logits to shared memory, and its settings ----
    // Position i of the stretch is logit first + i; the row's first logit lies `-first` past a 16-byte boundary in CTA 0.
    const T* const logits = static_cast<const T*>(p.logits) + row * p.row_stride;
    const int first = rank * p.stretch - (int)((reinterpret_cast<uintptr_t>(logits) & 15) / sizeof(T));
    // A warp's run: blocks [block0, block0 + run) of the stretch, the first `held` of them in shared memory.
    const int blocks = p.stretch / kBlock, block0 = blocks * warp / kSampleWarps, run = blocks * (warp + 1) / kSampleWarps - block0;
    const int held = p.held;
    const int from_e = first + block0 * kBlock + lane * 4;   // this lane's first logit
    T* const x_lane = x + warp * held * kBlock + lane * 4;
    // whether all of block j of the run are logits of the row
    auto inside = [&](int e0) { return e0 >= 0 && e0 + kBlock <= p.vocab; };
    for (int j = 0; j < min(held, run); ++j) {
        const int e = from_e + j * kBlock;
        if (inside(first + (block0 + j) * kBlock)) {
            if constexpr (sizeof(T) == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(x_lane + j * kBlock)), "l"(logits + e) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(x_lane + j * kBlock)), "l"(logits + e) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (e + i >= 0 && e + i < p.vocab) x_lane[j * kBlock + i] = logits[e + i];
                else store_logit(&x_lane[j * kBlock + i], -INFINITY);
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
    bool infinite = false;
    // this lane's four logits of block j of warp w's run
    auto quad_at = [&](int w, int j, float (&v)[4]) {
        const int b = blocks * w / kSampleWarps + j, e0 = first + b * kBlock, e = e0 + lane * 4;
        if (j < held || inside(e0)) {
            quad_of(j < held ? x + (w * held + j) * kBlock + lane * 4 : logits + e, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = e + i >= 0 && e + i < p.vocab ? load_logit(logits + e + i) : -INFINITY;
        }
        if (infinite && j >= held) {   // the infinite ones share the draw
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] == INFINITY ? 0.f : -INFINITY;
        }
    };
    auto far_quad = [&](int j, float (&v)[4]) {
        const int e0 = first + (block0 + j) * kBlock, e = from_e + j * kBlock;
        if (inside(e0)) {
            quad_of(logits + e, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = e + i >= 0 && e + i < p.vocab ? load_logit(logits + e + i) : -INFINITY;
        }
        if (infinite) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] == INFINITY ? 0.f : -INFINITY;
        }
    };
    // f(j, v) for every block of the warp's run; those in shared memory first, and without looking where they lie
    const int near = min(held, run);
    auto for_blocks = [&](auto f) {
#pragma unroll 2
        for (int j = 0; j < near; ++j) {
            float v[4];
            quad_of(x_lane + j * kBlock, v);
            f(j, v);
        }
#pragma unroll 1
        for (int j = near; j < run; j += kFar) {   // (the loads of a few blocks at once)
            float v[kFar][4];
#pragma unroll
            for (int i = 0; i < kFar; ++i)
                if (j + i < run) far_quad(j + i, v[i]);
#pragma unroll
            for (int i = 0; i < kFar; ++i)
                if (j + i < run) f(j + i, v[i]);
        }
    };

    // ---- the largest logit, and the cut ----
    float top = -INFINITY;
#pragma unroll 4
    for (int j = near; j < run; ++j) {
        float v[4];
        far_quad(j, v);
        top = max3(max3(top, v[0], v[1]), v[2], v[3]);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();   // (a warp copies its own run)
#pragma unroll 4
    for (int j = 0; j < near; ++j) {
        float v[4];
        quad_of(x_lane + j * kBlock, v);
        top = max3(max3(top, v[0], v[1]), v[2], v[3]);
    }
    top = fmaxf(top, -INFINITY);   // (NaN where all are)
    if (by_count || by_share) {
        // About `want` logits: enough that a cut somewhat too high still leaves k, or most rows' top-p, and few beside the room for kListed.
        // With so many above the cut, a share of 1 - exp(-want / threads) of the threads' tops is: the warp's q-th largest one of 32, from 0 on.
        const float want = by_count ? fmaxf(192.f, 1.5f * (float)top_k + 64.f) : 512.f;
        const int q = min(31, (int)(32.f * (1.f - __expf(-want / (float)(ranks * kSampleThreads)))));
        uint32_t key = key_of(top), most = __reduce_max_sync(0xffffffffu, key);
        top = value_of(most);
#pragma unroll 1
        for (int i = 0; i < q; ++i) {
            if (lane == __ffs(__ballot_sync(0xffffffffu, key == most)) - 1) key = 0;
            most = __reduce_max_sync(0xffffffffu, key);
        }
        const float cut = value_of(max(most, key_of(-INFINITY)));
        if (lane == 0) s.warp_top[warp] = top, s.warp_cut[warp] = cut;
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) s.warp_top[warp] = top;
    }
    __syncthreads();
    if (ranks > 1) cluster_wait();   // all CTAs of the row have started: their shared memory may be written
    if (warp == 0) {
        float t = lane < kSampleWarps ? s.warp_top[lane] : -INFINITY, cut = 0.f;
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
#pragma unroll 1
        for (int j = 0; j < run; ++j) {
            float v[4];
            quad_at(warp, j, v);
#pragma unroll
            for (int i = 3; i >= 0; --i)
                if (v[i] == m) at = min(at, (uint32_t)(from_e + j * kBlock + i));
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
    if (m == INFINITY) {
        infinite = true;
        m = cut = 0.f;
        for (int j = 0; j < near; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) store_logit(&x_lane[j * kBlock + i], load_logit(&x_lane[j * kBlock + i]) == INFINITY ? 0.f : -INFINITY);
    }

    // Temperatures at which no number but the largest logit has a weight are all alike: the next one lies 2^-24 of it below at least, and here 128 times the
    // temperature.
    const uint32_t m_key = key_of(m);
    const float below = fmaxf(value_of(m_key - 1), -FLT_MAX), t = fmaxf(temperature, fabsf(m) * 0x1p-31f);
    Weigh weigh;
    weigh.c = t == temperature ? usual_c : 16. * 1.4426950408889634 / (double)t;
    const double top_c = rint((double)m * weigh.c);
    weigh.shift = 6755399441055744.0 - top_c;
    if (tid < 16) {
        const double power = s.power[tid] * Weigh::power_of(top_c - (double)m * weigh.c);
        s.power[tid] = __hiloint2double(__double2hiint(power) - tid * 0x10000, __double2loint(power));
    }
    weigh.floor = fmaxf(fminf(below, m - 44.3614f * t), -FLT_MAX);   // 64 ln 2
    weigh.power = s.power;
    const bool low = weigh.floor == -FLT_MAX;   // then minus infinity and NaN have to be told from the floor
    __syncthreads();
    const uint64_t least = min_p > 0.f ? (uint64_t)ceil((double)fminf(min_p, 1.f) * (double)units_once(weigh.c, weigh.shift, weigh.floor, weigh.power, m)) : 0;
    auto block_sum = [&](uint64_t v) {   // (a barrier before the next one)
        v = warp_sum_u64(v);
        if (lane == 0) s.warp_sum[warp] = v;
        __syncthreads();
        return warp_sum_u64(lane < kSampleWarps ? s.warp_sum[lane] : 0);
    };
    // Adds four logits' units to four sums (of a run of 2^8 blocks at most, less than 2^52 units each).
    auto add_units = [&](const float (&v)[4], double (&sum)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double to = weigh.add(v[i], sum[i]);
            sum[i] = !low || v[i] > -INFINITY ? to : sum[i];
        }
    };
    auto units_of = [&](const double (&sum)[4]) { return (Weigh::units(sum[0]) + Weigh::units(sum[1])) + (Weigh::units(sum[2]) + Weigh::units(sum[3])); };
    // (Parts whose sums over a stretch fit 32 bits: a sum in two halves needs what was there before for its carry, and waits for it.)
    auto add_to_bin = [&](int buf, int at, uint64_t u) {
        atomicAdd(&s.bins[buf][0][at], 1u);
        atomicAdd(&s.bins[buf][1][at], (uint32_t)u & 0x7fffu);
        atomicAdd(&s.bins[buf][2][at], (uint32_t)(u >> 15) & 0x7fffu);
        if (u >> 30) atomicAdd(&s.bins[buf][3][at], (uint32_t)(u >> 30));
    };
    auto clear_bins = [&](int buf) {
        if (tid < kSampleBins)
#pragma unroll
            for (int i = 0; i < 4; ++i) s.bins[buf][i][tid] = 0;
    };
    auto units_at = [&](float v) { return units_once(weigh.c, weigh.shift, weigh.floor, weigh.power, v); };
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
    int tie_to = -1;   // or those up to this index, whatever their number
    if (by_count || by_share) {
        // ---- the logits above the cut, collected in one CTA ----
        uint64_t total = 0, above = 0;
        const int most = kListed / ranks;   // of a CTA (ranks: a power of two)
        uint2* const mine = s.listed + rank * most;
        auto list = [&](const float (&v)[4], int j) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] >= cut && v[i] > -INFINITY) {
                    const uint32_t at = atomicAdd(&s.num_mine, 1u);
                    if (at < most) mine[at] = make_uint2(__float_as_uint(v[i]), (uint32_t)(from_e + j * kBlock + i));
                }
        };
        const int collector = row % ranks;
        // The CTA's part to the collecting CTA; returns the units of what this thread had of it where they are asked for.
        auto hand_over = [&](bool weighed) {
            uint64_t w = 0;
            for (int i = tid; i < (int)min(s.num_mine, (uint32_t)most); i += kSampleThreads) {
                const uint2 e = mine[i];
                if (rank != collector) cluster.map_shared_rank(&s, collector)->listed[rank * most + i] = e;
                if (weighed) w += units_at(__uint_as_float(e.x));
            }
            return w;
        };
        if (by_share && !by_count) {
            double sums[4] = {Weigh::kZero, Weigh::kZero, Weigh::kZero, Weigh::kZero};
            for_blocks([&](int j, const float (&v)[4]) {
                add_units(v, sums);
                if (max4(v) >= cut) list(v, j);
            });
            total = block_sum(units_of(sums));
        } else {
            for_blocks([&](int j, const float (&v)[4]) {
                if (max4(v) >= cut) list(v, j);
            });
        }
        __syncthreads();
        const uint32_t listed = s.num_mine;
        above = hand_over(!by_count);
        if (!by_count) above = block_sum(above);   // (of those that are listed)
        if (warp == 0 && lane < ranks) {
            SampleShared* peer = cluster.map_shared_rank(&s, lane);
            peer->rank_listed[rank] = listed;
            peer->rank_total[rank] = total;
            peer->rank_above[rank] = above;
        }
        all_here();
        uint32_t n = lane < ranks ? s.rank_listed[lane] : 0;
        const bool fits = __all_sync(0xffffffffu, n <= most);
        n = __reduce_add_sync(0xffffffffu, n);
        uint64_t all = 0, target = top_k;
        if (!by_count) {
            all = warp_sum_u64(lane < ranks ? s.rank_total[lane] : 0);
            above = warp_sum_u64(lane < ranks ? s.rank_above[lane] : 0);
            target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), all, true));
        }
        const bool direct = fits && (by_count ? n : above) >= target;
        bool listed_window = false;
        uint32_t window_lo = 0, window_hi = 0;   // keys among which the threshold may lie, where they were too many for a list
        uint64_t window_above = 0;
        uint32_t low_key = min(key_of(cut), m_key);   // of what is collected
        if (direct && rank != collector) return;
        if (!direct && fits && !by_count && cut > -FLT_MAX) {
            // -- about where the threshold lies: an eighth of the blocks below the cut, in 256 bins of equal width
            Interval iv;
            iv.over(kLowestKey, max(key_of(cut), kLowestKey + 1) - 1, weigh.floor);
            __syncthreads();
            clear_bins(0);
            __syncthreads();
            const int step = min(8, max(2, run));
            const float first_v = value_of(iv.lo);
            const int drop = max(0, 64 - __clzll((long long)units_at(cut)) - 19);   // 19 bits of a weight: sums of 8192 of them fit 32
#pragma unroll 1
            for (int j = step / 2; j < run; j += step) {
                float v[4];
                quad_at(warp, j, v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (v[i] >= first_v && v[i] < cut) atomicAdd(&s.bins[0][0][iv.bin(v[i], 0)], (uint32_t)(units_at(v[i]) >> drop));
            }
            all_here();
            uint64_t w = 0;
            if (tid < kSampleBins) {
                uint32_t part[kSampleRanks];
#pragma unroll
                for (int r = 0; r < kSampleRanks; ++r) part[r] = cluster.map_shared_rank(&s, min(r, ranks - 1))->bins[0][0][kSampleBins - 1 - tid];
#pragma unroll
                for (int r = 0; r < kSampleRanks; ++r) w += r < ranks ? part[r] : 0;
            }
            pick(s, 0, w, 0, 0, true, ~0ull);   // (everything)
            const double sampled = (double)s.found.above_w, rest = (double)(all - above);
            pick(s, 0, w, 0, 0, true, (uint64_t)fmax(1., fmin(sampled, ceil(sampled * ((double)(target - above) / rest)))));
            const auto f = s.found;
            listed_window = sampled > 0. && f.bin >= 0 && f.w > 0;
            if (listed_window) {   // (the same in all CTAs)
                const double in_bin = (sampled * ((double)(target - above) / rest) - (double)f.above_w) / (double)f.w;
                const double density = (double)f.w / sampled * rest * (double)iv.per;   // units per unit of x
                // -- the units above three places, a fiftieth of the rest apart
                const float apart = (float)(0.02 * rest / density), mid = iv.x_lo + ((float)(f.bin + 1) - (float)in_bin) / iv.per;
                const float place[3] = {fminf(mid + apart, cut), mid, fmaxf(mid - apart, -FLT_MAX)};
                double sums[3][2];
#pragma unroll
                for (int i = 0; i < 3; ++i) sums[i][0] = sums[i][1] = Weigh::kZero;
#pragma unroll 1
                for (int j = 0; j < run; ++j) {
                    float v[4];
                    if (j < held) quad_of(x_lane + j * kBlock, v);
                    else quad_at(warp, j, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        double a, b;
                        weigh.factors(v[i], a, b);
#pragma unroll
                        for (int c = 0; c < 3; ++c) {
                            const double to = fma(a, b, sums[c][i & 1]);
                            sums[c][i & 1] = v[i] >= place[c] ? to : sums[c][i & 1];
                        }
                    }
                }
                uint64_t sum[3];
#pragma unroll
                for (int c = 0; c < 3; ++c) {
                    __syncthreads();
                    sum[c] = block_sum(Weigh::units(sums[c][0]) + Weigh::units(sums[c][1]));
                }
                if (warp == 0 && lane < ranks) {
                    SampleShared* peer = cluster.map_shared_rank(&s, lane);
#pragma unroll
                    for (int c = 0; c < 3; ++c) peer->rank_places[rank][c] = sum[c];
                }
                if (tid == 0) s.num_mine = 0;
                all_here();
                double miss[3];   // units by which the target lies further
#pragma unroll
                for (int c = 0; c < 3; ++c) miss[c] = (double)(int64_t)(target - warp_sum_u64(lane < ranks ? s.rank_places[lane][c] : 0));
                // the place where nothing is missed, by the parabola through the three; within their width either way
                const double d01 = (place[1] - place[0]) / (miss[1] - miss[0]), d12 = (place[2] - place[1]) / (miss[2] - miss[1]);
                const double d012 = (d12 - d01) / (miss[2] - miss[0]);
                double at = place[0] - miss[0] * d01 + miss[0] * miss[1] * d012;
                if (!(at > place[2] - apart)) at = place[2] - apart;
                if (!(at < place[0] + apart)) at = place[0] + apart;
                // -- some hundreds of logits around it, and the units above them
                const double each = (double)units_at((float)at) + 1., wide = 320. * each / fmax(density, 1.);
                const float hi_v = (float)(at + wide), lo_v = fminf((float)(at - wide), hi_v);
                sums[0][0] = sums[0][1] = Weigh::kZero;
#pragma unroll 1
                for (int j = 0; j < run; ++j) {
                    float v[4];
                    if (j < held) quad_of(x_lane + j * kBlock, v);
                    else quad_at(warp, j, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const double to = weigh.add(v[i], sums[0][i & 1]);
                        sums[0][i & 1] = v[i] > hi_v ? to : sums[0][i & 1];
                        if (v[i] >= lo_v && v[i] <= hi_v && v[i] > -INFINITY) {
                            const uint32_t to_at = atomicAdd(&s.num_mine, 1u);
                            if (to_at < most) mine[to_at] = make_uint2(__float_as_uint(v[i]), (uint32_t)(from_e + j * kBlock + i));
                        }
                    }
                }
                sum[0] = block_sum(Weigh::units(sums[0][0]) + Weigh::units(sums[0][1]));
                const uint32_t found = s.num_mine;
                uint64_t found_w = hand_over(true);
                __syncthreads();
                found_w = block_sum(found_w);
                if (warp == 0 && lane < ranks) {
                    SampleShared* peer = cluster.map_shared_rank(&s, lane);
                    peer->rank_listed[rank] = found;
                    peer->rank_total[rank] = sum[0];
                    peer->rank_above[rank] = found_w;
                }
                all_here();
                const uint64_t over = warp_sum_u64(lane < ranks ? s.rank_total[lane] : 0), among = warp_sum_u64(lane < ranks ? s.rank_above[lane] : 0);
                const bool all_listed = __all_sync(0xffffffffu, lane >= ranks || s.rank_listed[lane] <= most);
                listed_window = all_listed && over < target && over + among >= target;
                if (listed_window) {
                    target -= over;
                    low_key = key_of(lo_v);
                } else if (over < target && lo_v <= hi_v) {
                    window_lo = max(key_of(lo_v), kLowestKey);
                    window_hi = min(key_of(hi_v), m_key);
                    window_above = over;
                }
            }
        }
        if ((direct || listed_window) && rank == collector) {
            uint32_t key[kHeld], order[kHeld];   // order: falls with the index
            uint64_t units[kHeld];
            unsigned live = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                const int at = tid + i * kSampleThreads, r = at / most;
                key[i] = order[i] = 0;
                units[i] = 0;
                if (at - r * most < (int)s.rank_listed[r]) {
                    const uint2 e = s.listed[at];
                    key[i] = key_of(__uint_as_float(e.x));
                    order[i] = ~e.y;
                    units[i] = units_at(__uint_as_float(e.x));
                    live |= 1u << i;
                }
            }
            __syncthreads();
            clear_bins(0);
            auto live_units = [&](unsigned of) {
                uint64_t sum = 0;
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (of >> i & 1) sum += units[i];
                __syncthreads();
                return block_sum(sum);
            };
            // Five steps of one kind: of some logits, in falling order of their key or of `order`, those are left that reach a target of number or weight.
            // 0: top-k; 1: of equal ones at its threshold the first; 2, 3: top-p likewise; 4: the token, the last of those that the draw takes to reach.
            uint64_t kept = 0;   // units of what is left (0: not known)
            unsigned equal = 0;
#pragma unroll 1
            for (int step = by_count ? 0 : 2; step < (direct ? 5 : 4); ++step) {
                if (step == 0 && n <= (uint32_t)top_k) step = 2;
                if (step == 2) {
                    if (by_count && by_share) target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), kept ? kept : live_units(live), true));
                    if (!by_share) step = 4;
                }
                if (step == 4) {
                    if (least > 0) {
                        kept = 0;
#pragma unroll
                        for (int i = 0; i < kHeld; ++i)
                            if (units[i] < least) live &= ~(1u << i);
                    }
                    if (kept == 0) kept = live_units(live);
                    target = draw_of(kept) + 1;
                }
                const bool by_index = step == 1 || step >= 3, by_weight = step == 2 || step == 4;
                uint32_t lo = by_index ? ~(uint32_t)(p.vocab - 1) : low_key, hi = by_index ? ~0u : m_key, above_n = 0;
                uint64_t above_w = 0;
                unsigned of = step == 1 || step == 3 ? equal : live;
                SampleShared::Found f;
#pragma unroll 1
                for (;;) {   // 256 bins a pass, until the one where the target is reached has one logit, or one key, or (by number) is kept whole
                    const int shift = max(by_index ? 0 : kGrain<T>, 24 - __clz(hi - lo));
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < kHeld; ++i) {
                        const uint32_t k = by_index ? order[i] : key[i];
                        if (of >> i & 1 && k >= lo && k <= hi) add_to_bin(0, (int)((k - lo) >> shift), units[i]);
                    }
                    __syncthreads();
                    uint32_t bin_n = 0;
                    uint64_t bin_w = 0;
                    if (tid < kSampleBins) {   // (and the bin is ready for the next pass)
                        const int at = kSampleBins - 1 - tid;
                        bin_n = s.bins[0][0][at];
                        bin_w = ((uint64_t)s.bins[0][3][at] << 30) + ((uint64_t)s.bins[0][2][at] << 15) + s.bins[0][1][at];
#pragma unroll
                        for (int i = 0; i < 4; ++i) s.bins[0][i][at] = 0;
                    }
                    pick(s, bin_n, bin_w, above_n, above_w, by_weight, target);
                    f = s.found;
                    above_n = f.above_n;
                    above_w = f.above_w;
                    lo += (uint32_t)f.bin << shift;
                    hi = lo + min(hi - lo, (1u << shift) - 1);
                    if (!by_index && shift == kGrain<T>) lo = hi = only_key<T>(lo);
                    if (lo == hi || f.n == 1 || (!by_weight && (direct || !by_index) && above_n + f.n == target)) break;
                }
                if (step == 4) {
#pragma unroll
                    for (int i = 0; i < kHeld; ++i)
                        if (live >> i & 1 && order[i] >= lo && order[i] <= hi) emit((int)~order[i], units[i], kept);
                    break;
                }
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if ((by_index ? order[i] : key[i]) < lo) of &= ~(1u << i);
                if (by_index) {
                    live |= of;
                    if (!direct && tid < ranks) cluster.map_shared_rank(&s, tid)->front[2] = ~lo;   // (the last of them: the search ends at a single one)
                    continue;
                }
                live = of;
                uint32_t take = f.n;
                const uint64_t each = f.n > 1 ? f.w / f.n : f.w;
                if (!by_weight) take = (uint32_t)(target - above_n);
                else if (f.n > 1 && each > 0) take = (uint32_t)min((uint64_t)f.n, (target - above_w + each - 1) / each);
                kept = above_w + (take == f.n ? f.w : take * each);
                if (!direct && tid < ranks) {
                    SampleShared* peer = cluster.map_shared_rank(&s, tid);
                    peer->front[0] = take == f.n ? lo : lo + 1;
                    peer->front[1] = take == f.n ? 0 : lo;
                }
                if (take == f.n) {
                    ++step;   // (none of equal ones are left out)
                    continue;
                }
                equal = 0;
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (live >> i & 1 && key[i] == lo) equal |= 1u << i;
                live &= ~equal;
                target = take;
            }
            if (direct) return;
        }
        all_here();   // (with the front part, or all have read the bins that told nothing)
        if (listed_window) {
            keep = s.front[0];
            if (s.front[1] != 0) {
                tie_key = s.front[1];
                tie_to = (int)s.front[2];
            }
        } else {

        // ---- the threshold lies lower: the lowest key that is kept whole, and how many logits of the key in front of it, by all CTAs ----
        clear_bins(0);
        clear_bins(1);
        __syncthreads();
        // the lowest key of the linear interval's bin `bin` (one past the last where there is none): the bin of a number never falls
        auto edge_of = [&](const Interval& iv, int bin) {
            uint32_t a = iv.lo, b = iv.hi + 1;
#pragma unroll 1
            while (a < b) {
                const uint32_t mid = a + (b - a) / 2;
                if (iv.bin(value_of(mid), mid) >= bin) b = mid;
                else a = mid + 1;
            }
            return a;
        };
        auto edges = [&](const Interval& iv, int bin_lo, int bin_hi) {   // to s.edge: the lowest keys of a bin and of another one
            if (lane == 0 && warp < 2) s.edge[warp] = edge_of(iv, warp ? bin_hi : bin_lo);
            __syncthreads();
        };
        // The search: of the logits from key `bottom` on the front part is kept that reaches `target` logits, or units; above_n and above_w lie above the interval.
        bool by_weight = !by_count;
        const uint32_t cut_key = max(kLowestKey, key_of(cut));
        uint32_t bottom = kLowestKey, above_n = 0;
        uint64_t above_w = 0;
        if (!by_count) target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), all, true));
        Interval iv;
        if (window_lo != 0 && window_lo <= window_hi) {
            iv.by_key(window_lo, window_hi, kGrain<T>);
            above_w = window_above;
        } else {
            iv.by_key(cut_key, m_key, kGrain<T>);
        }
#pragma unroll 1
        for (int pass = 0;; ++pass) {
            // bins of the interval's logits, summed over the cluster
            const int buf = pass & 1;
            if (pass >= 2) {   // (its bins of two passes ago have been read: a barrier lies between)
                clear_bins(buf);
                __syncthreads();
            }
            uint32_t bin_n = 0;
            uint64_t bin_w = 0;
            {
                const float from = value_of(iv.lo), to = value_of(iv.hi);
#pragma unroll 1
                for (int j = 0; j < run; ++j) {
                    float v[4];
                    quad_at(warp, j, v);
                    bool any = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) any |= v[i] >= from && v[i] <= to;
                    if (!any) continue;
                    uint64_t u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] = weigh(v[i]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t key = key_of(v[i]);
                        if (v[i] >= from && key >= iv.lo && key <= iv.hi) add_to_bin(buf, iv.bin(v[i], key), u[i]);
                    }
                }
                all_here();
                if (tid < kSampleBins) {
                    const int at = kSampleBins - 1 - tid;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t part[kSampleRanks];
#pragma unroll
                        for (int r = 0; r < kSampleRanks; ++r) part[r] = cluster.map_shared_rank(&s, min(r, ranks - 1))->bins[buf][i][at];   // (all on their way at once)
                        uint64_t sum = 0;
#pragma unroll
                        for (int r = 0; r < kSampleRanks; ++r) sum += r < ranks ? part[r] : 0;
                        if (i == 0) bin_n = (uint32_t)sum;
                        else bin_w += sum << 15 * (i - 1);
                    }
                }
            }
            pick(s, bin_n, bin_w, above_n, above_w, by_weight, target);
            const auto f = s.found;
            above_n = f.above_n;
            above_w = f.above_w;
            bool done = true;
            if (f.bin < 0) {
                if (iv.lo > bottom) {
                    iv.over(bottom, iv.lo - 1, weigh.floor);
                    done = false;
                } else {   // everything from there on, and of what was kept of the key in front of it
                    keep = bottom;
                    if (ties > 0) {
                        const uint64_t w = max((uint64_t)1, units_at(value_of(tie_key)));
                        ties = (uint32_t)min((uint64_t)ties, target <= above_w ? 0 : (target - above_w + w - 1) / w);
                    }
                }
            } else if (!iv.linear && iv.shift == kGrain<T>) {   // one key, of equal weights
                const uint32_t key = only_key<T>(iv.lo + ((uint32_t)f.bin << iv.shift));
                const uint64_t w = max((uint64_t)1, f.w / f.n);
                const uint32_t take = (uint32_t)(by_weight ? min((uint64_t)f.n, f.w == 0 ? f.n : (target - above_w + w - 1) / w) : target - above_n);
                tie_key = key;
                ties = take == f.n ? 0 : take;
                tie_before = 0;
                for (int r = 0; r < rank; ++r) tie_before += cluster.map_shared_rank(&s, r)->bins[buf][0][f.bin];
                keep = take == f.n ? key : key + 1;
                above_w += take == f.n ? f.w : take * w;
            } else {
                uint32_t lo = iv.lo + (iv.linear ? 0 : (uint32_t)f.bin << iv.shift), hi = lo + min(iv.hi - lo, (1u << iv.shift) - 1);
                if (iv.linear) {
                    edges(iv, f.bin, f.bin + 1);
                    lo = s.edge[0];
                    hi = s.edge[1] - 1;
                }
                if (by_weight ? f.n == 1 : above_n + f.n == target) {
                    keep = lo;
                    ties = 0;
                    above_w += f.w;
                } else {
                    iv.by_key(lo, hi, kGrain<T>);
                    done = false;
                }
            }
            if (!done) continue;
            if (by_weight || !by_share) break;
            // top-p of what top-k has left (above_w units)
            by_weight = true;
            target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), above_w, true));
            if (keep > m_key) {   // all of it are equal
                const uint64_t w = units_at(value_of(tie_key));
                ties = (uint32_t)min((uint64_t)ties, (target + w - 1) / w);
                break;
            }
            bottom = keep;
            above_n = 0;
            above_w = 0;
            iv.by_key(keep, m_key, kGrain<T>);
        }
        }
    }

    // ---- the kept weights' sums ----
    const float tie = value_of(tie_key);
    uint32_t tie_at = 0;   // ties in front of the warp's next block
    if (ties > 0) {
        uint32_t n = 0;
#pragma unroll 1
        for (int j = 0; j < run; ++j) {
            float v[4];
            quad_at(warp, j, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) n += v[i] == tie;
        }
        n = __reduce_add_sync(0xffffffffu, n);
        __syncthreads();
        if (lane == 0) s.warp_word[warp] = n;
        __syncthreads();
        tie_at = tie_before;
        for (int w = 0; w < warp; ++w) tie_at += s.warp_word[w];
    }
    // No logit below this one is kept: of the threshold, or of min_p (less what the rounding of its place can be off).
    float from = value_of(ties > 0 || tie_to >= 0 ? tie_key : keep);
    if (least > 0) from = fmaxf(from, fmaxf(-FLT_MAX, m + t * logf(fminf(min_p, 1.f)) * 1.0001f - 1e-5f * (fabsf(m) + t)));
    // units of four neighbouring logits from index e on, none where they are not kept; `at`: ties so far, moved on
    auto kept_units = [&](const float (&v)[4], int e, uint32_t& at, uint64_t (&w)[4]) {
        bool in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i] = v[i] >= from && (key_of(v[i]) >= keep || (v[i] == tie && e + i <= tie_to));
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
    if (ties == 0 && tie_to < 0 && least == 0) {
        double sums[4] = {Weigh::kZero, Weigh::kZero, Weigh::kZero, Weigh::kZero};
        for_blocks([&](int, const float (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double to = weigh.add(v[i], sums[i]);
                sums[i] = v[i] >= from ? to : sums[i];
            }
        });
        sum = units_of(sums);
    } else {
        uint32_t at = tie_at;
#pragma unroll 1
        for (int j = 0; j < run; ++j) {
            float v[4];
            uint64_t w[4];
            quad_at(warp, j, v);
            if (ties == 0 && !__any_sync(0xffffffffu, max4(v) >= from)) continue;
            kept_units(v, from_e + j * kBlock, at, w);
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
    const uint64_t rank_sum = lane < ranks ? s.rank_kept[lane] : 0, total = warp_sum_u64(rank_sum);
    uint64_t in_front = warp_sum_u64(lane < rank ? rank_sum : 0);
    const uint64_t drawn = draw_of(total);
    if (drawn < in_front || drawn >= in_front + s.rank_kept[rank]) return;
    // The warps look through the run of the one that it falls into, a block each.
    int of = 0;
    for (uint64_t w = s.warp_sum[0]; in_front + w <= drawn; w = s.warp_sum[of]) {
        in_front += w;
        ++of;
    }
    const int of_block0 = blocks * of / kSampleWarps, of_run = blocks * (of + 1) / kSampleWarps - of_block0;
    for (int round = 0; round < of_run; round += kSampleWarps) {
        const int j = round + warp;
        uint64_t w[4] = {0, 0, 0, 0};
        if (j < of_run) {
            float v[4];
            uint32_t at = tie_before;
            if (ties > 0) {   // those in front of the block
                uint32_t n = 0;
                for (int c = 0; c < j; ++c) {
                    quad_at(of, c, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) n += v[i] == tie;
                }
                at += __reduce_add_sync(0xffffffffu, n);
                for (int c = 0; c < of; ++c) at += s.warp_word[c];
            }
            quad_at(of, j, v);
            kept_units(v, first + (of_block0 + j) * kBlock + lane * 4, at, w);
        }
        const uint64_t here = (w[0] + w[1]) + (w[2] + w[3]), up_to = warp_scan_u64(here, lane);
        if (round > 0) __syncthreads();
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
            emit(first + (of_block0 + j) * kBlock + lane * 4 + i, i == 0 ? w[0] : i == 1 ? w[1] : i == 2 ? w[2] : w[3], total);
        }
        for (int c = 0; c < kSampleWarps; ++c) in_front += s.block[c];
    }
}

static_assert((kMaxVocab + 8 + kSampleRanks * kBlock) / kSampleRanks < 1 << 16, "parts of a bin's sum fit 32 bits");
constexpr int sample_smem(int ctas) { return ctas == 1 ? 227 * 1024 : 228 * 1024 / ctas - 1024; }   // of a CTA
static_assert(sample_smem(3) - sizeof(SampleShared) >= 64 * 1024, "what is left of a third of an SM's shared memory is 16384 logits of 32 bits");

template <class T>
cudaError_t configure_sample() {
    cudaError_t e = cudaFuncSetAttribute(sw_sample_kernel<T, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, sample_smem(1));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(sw_sample_kernel<T, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, sample_smem(2));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(sw_sample_kernel<T, 3>, cudaFuncAttributeMaxDynamicSharedMemorySize, sample_smem(3));
    return e;
}
cudaError_t configure_sample_kernels() {
    cudaError_t e = configure_sample<float>();
    if (e == cudaSuccess) e = configure_sample<__nv_bfloat16>();
    if (e == cudaSuccess) e = configure_sample<__half>();
    return e;
}

cudaError_t launch_sample(const SampleParams& params, int dtype, int num_sms, cudaStream_t stream) {
    SampleParams p = params;
    const int size = dtype == SW_DTYPE_F32 ? 4 : 2;
    // CTAs of a row: as many as give each 16384 logits at most (64 KB: three CTAs an SM), and more where rows are few.
    const int64_t positions = (int64_t)p.vocab + 16 / size - 1;   // (a row may start anywhere behind a 16-byte boundary)
    int ranks = 1;
    while (ranks < kSampleRanks && (positions > ranks * 16384 || (p.rows * ranks < num_sms && positions > ranks * 2048))) ranks *= 2;
    p.stretch = (int)((positions + ranks * kBlock - 1) / (ranks * kBlock) * kBlock);
    const int ctas = p.rows * ranks > 2 * num_sms ? 3 : p.rows * ranks > num_sms || p.stretch < 4096 ? 2 : 1, warps = (ctas == 1 ? kThreadsFor<1> : kThreadsFor<2>) / 32;
    const int run = (p.stretch / kBlock + warps - 1) / warps;   // blocks of the longest run
    const int room = (sample_smem(ctas) - (int)sizeof(SampleShared)) / (warps * kBlock * size);
    p.held = room < run ? room : run;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * ranks));
    cfg.blockDim = dim3(warps * 32);
    cfg.dynamicSmemBytes = sizeof(SampleShared) + (size_t)p.held * warps * kBlock * size;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    auto launch = [&](auto* one, auto* two, auto* three) { return cudaLaunchKernelEx(&cfg, ctas == 1 ? one : ctas == 2 ? two : three, p); };
    if (dtype == SW_DTYPE_F32) return launch(sw_sample_kernel<float, 1>, sw_sample_kernel<float, 2>, sw_sample_kernel<float, 3>);
    if (dtype == SW_DTYPE_BF16) return launch(sw_sample_kernel<__nv_bfloat16, 1>, sw_sample_kernel<__nv_bfloat16, 2>, sw_sample_kernel<__nv_bfloat16, 3>);
    return launch(sw_sample_kernel<__half, 1>, sw_sample_kernel<__half, 2>, sw_sample_kernel<__half, 3>);
}

}  // namespace sw
