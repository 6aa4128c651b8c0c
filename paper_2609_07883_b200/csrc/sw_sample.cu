// The draw of one token a row from logits: temperature, top-k, top-p and min-p, by a given uniform number.
//
// Weights are w = exp((x - max) / temperature).  All three limits keep a front part of the logits in falling order (equal ones by index), so what
// they leave is known by one threshold and a number of elements at it, and nothing is sorted.  The token is the first, by index, up to which the
// kept weights sum to more than u times their total.
//
// A border between tokens, or of top-p, is a sum over all logits: with 128256 about equal ones, sums in fp32 would put every tenth draw on the wrong side.
// Weights are worked out in 64 bits (2^x from a table of 32 powers and a polynomial of degree four, 8e-14 off) and rounded to 2^-44 of the
// largest; their sums are integers, exact in any order, and equal logits have equal weights.
//
// A cluster of 1 to 8 CTAs has a row; each CTA keeps an equal stretch in shared memory as fp32, so logits are read from memory once.  Then
//   - the row's largest logit, and a cut below which most logits lie: a quantile of the threads' largest ones (its median over warps and CTAs).  It
//     only has to be about right;
//   - top-k, top-p: the threshold by radix, 256 bins a pass with their number of logits and weight, over the logits above the cut; the CTAs read
//     one another's bins.  Where the threshold lies lower, 256 bins of equal width over the rest come first;
//   - the sums of the kept weights of every warp's run of logits; the CTA and the warp that the draw falls into look for the token.
// Bound by the logits' bytes, and by 64-bit arithmetic where all weights are needed (nine operations a logit).
#include <cfloat>
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "sw_mixed.cuh"

namespace sw {
namespace cg = cooperative_groups;

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32, kSampleBins = 256, kSampleRanks = 8;
constexpr int kBlock = 128;   // logits that a warp takes at once
constexpr uint32_t kLowestKey = 0x00800000u;   // ordered() of the lowest finite number
constexpr int kUnitBits = 44;                  // the largest weight is 2^44 units: sums of up to 2^19 of them fit 63 bits

struct SampleShared {
    uint32_t count[2][kSampleBins], low[2][kSampleBins], high[2][kSampleBins];   // by the parity of the pass: logits, and units in two halves
    uint64_t weight[kSampleBins];                                                // summed over the cluster
    uint32_t number[kSampleBins], before[kSampleBins];                           // likewise; of the CTAs before this one
    double power[32];                                                            // 2^(j / 32)
    uint64_t rank_total[kSampleRanks], rank_kept[kSampleRanks], warp_sum[kSampleWarps];
    float rank_top[kSampleRanks], rank_cut[kSampleRanks], warp_top[kSampleWarps], warp_cut[kSampleWarps];
    uint32_t rank_first[kSampleRanks], warp_word[kSampleWarps];
    struct {
        uint64_t above_w, w;
        uint32_t above_n, n, before;
        int bin;
    } found;
    uint32_t edge[2];
    alignas(16) float x[];
};

// Floats as integers of the same order (no NaN gets here); -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// A logit's weight in units.
struct Weigh {
    double c, mc;        // 32 / ln 2 / temperature, and times the largest logit
    float floor;         // weights below 2^-64 are none
    const double* power;
    __device__ __forceinline__ uint64_t operator()(float x) const {
        const double magic = 6755399441055744.0;   // 1.5 2^52: a sum with it is rounded to an integer, which its low word holds
        const double t = fma((double)fmaxf(x, floor), c, -mc), r = t + magic, f = t - (r - magic);
        const int n = __double2loint(r);
        const double q = fma(fma(fma(fma(9.172517872816247e-09, f, 1.6938633901956802e-06), f, 0.00023459619822185958), f, 0.021660849391722196), f,
                             0.9999999999999993);   // 2^(f / 32), |f| <= 1/2
        const double s = power[n & 31];
        const double scale = __hiloint2double(__double2hiint(s) + ((n >> 5) + kUnitBits) * 0x100000, __double2loint(s));
        return (uint64_t)__double_as_longlong(fma(q, scale, 4503599627370496.0)) - 0x4330000000000000ull;   // (2^52 likewise)
    }
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
// the value that `half` of the first n lanes' values lie above
__device__ __forceinline__ float lanes_median(float v, int n, int lane) {
    int above = 0;
    for (int j = 0; j < n; ++j) {
        const float o = __shfl_sync(0xffffffffu, v, j);
        above += o > v || (o == v && j < lane);
    }
    const unsigned at = __ballot_sync(0xffffffffu, lane < n && above == n / 2);
    return __shfl_sync(0xffffffffu, v, __ffs(at) - 1);
}

template <class T>
struct Vec;   // 16 bytes of logits as fp32
template <>
struct Vec<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ void widen(uint4 v, float (&f)[4]) {
        f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float one(float x) { return x; }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ void widen(uint4 v, float (&f)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
};
template <>
struct Vec<__half> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ void widen(uint4 v, float (&f)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = h.x, f[2 * i + 1] = h.y;
        }
    }
    static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
};

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

template <class T>
__global__ void __launch_bounds__(kSampleThreads, 2) sw_sample_kernel(const SampleParams p) {
    extern __shared__ __align__(16) unsigned char sample_raw[];
    SampleShared& s = *reinterpret_cast<SampleShared*>(sample_raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = (int)blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < 32) s.power[tid] = exp2((double)tid / 32.);
    for (int i = tid; i < 2 * kSampleBins; i += kSampleThreads) (&s.count[0][0])[i] = (&s.low[0][0])[i] = (&s.high[0][0])[i] = 0;
    grid_launch_dependents();
    grid_dependency_wait();
    auto all_here = [&] {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };

    // ---- the row's settings, and its logits to shared memory ----
    const float temperature = p.temperature ? p.temperature[row] : 1.f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    const bool greedy = !(temperature > 0.f), by_count = !greedy && top_k > 0 && top_k < p.vocab, by_share = !greedy && top_p < 1.f;
    // Position i of the stretch is logit first + i; the row's first logit lies `first` past a 16-byte boundary in CTA 0.
    constexpr int kN = Vec<T>::kN;
    const T* logits = static_cast<const T*>(p.logits) + row * p.row_stride;
    const int first = rank * p.stretch - (int)((reinterpret_cast<uintptr_t>(logits) & 15) / sizeof(T));
    float top = -INFINITY;
#pragma unroll 4
    for (int v = tid; v < p.stretch / kN; v += kSampleThreads) {
        const int e = first + v * kN;
        float f[kN];
        if (e >= 0 && e + kN <= p.vocab) {
            Vec<T>::widen(__ldcs(reinterpret_cast<const uint4*>(logits + e)), f);
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) f[i] = e + i >= 0 && e + i < p.vocab ? Vec<T>::one(logits[e + i]) : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            f[i] = fmaxf(f[i], -INFINITY);   // NaN counts as minus infinity
            top = fmaxf(top, f[i]);
        }
#pragma unroll
        for (int i = 0; i < kN; i += 4) *reinterpret_cast<float4*>(&s.x[v * kN + i]) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
    }

    // ---- the largest logit, and the cut ----
    if (by_count || by_share) {
        // the warp's 32 tops in falling order
#pragma unroll
        for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
            for (int j = k >> 1; j > 0; j >>= 1) {
                const float o = __shfl_xor_sync(0xffffffffu, top, j);
                top = ((lane & j) == 0) == ((lane & k) == 0) ? fmaxf(top, o) : fminf(top, o);
            }
        // above its q-th lie about q / 32 of the cluster's threads' tops, and a logit each at least
        const int q = by_count ? min(31, (2 * min(top_k, 1 << 16) + 64) * 32 / (ranks * kSampleThreads) + 1) : 4;
        const float cut = __shfl_sync(0xffffffffu, top, q);
        if (lane == 0) s.warp_top[warp] = top, s.warp_cut[warp] = cut;
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) s.warp_top[warp] = top, s.warp_cut[warp] = top;
    }
    __syncthreads();
    if (warp == 0) {
        float t = lane < kSampleWarps ? s.warp_top[lane] : -INFINITY;
        const float cut = lanes_median(lane < kSampleWarps ? s.warp_cut[lane] : -INFINITY, min(kSampleWarps, (p.stretch / kN + 31) / 32), lane);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
        if (lane < ranks) {
            SampleShared* to = cluster.map_shared_rank(&s, lane);
            to->rank_top[rank] = t;
            to->rank_cut[rank] = cut;
        }
    }
    all_here();
    float m = lane < ranks ? s.rank_top[lane] : -INFINITY;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = __shfl_sync(0xffffffffu, m, 0);
    float cut = lanes_median(lane < ranks ? s.rank_cut[lane] : -INFINITY, ranks, lane);
    if (m == -INFINITY) {   // nothing to draw from
        if (rank == 0 && tid == 0) {
            p.tokens[row] = -1;
            if (p.log_probs) p.log_probs[row] = -INFINITY;
        }
        return;
    }
    const float4* x4 = reinterpret_cast<const float4*>(s.x);
    if (m == INFINITY) {   // the infinite ones share the draw
        for (int i = tid; i < p.stretch; i += kSampleThreads) s.x[i] = s.x[i] == INFINITY ? 0.f : -INFINITY;
        m = cut = 0.f;
        __syncthreads();
    }
    const int blocks = p.stretch / kBlock, block0 = blocks * warp / kSampleWarps, block1 = blocks * (warp + 1) / kSampleWarps;   // of this warp

    if (greedy) {
        uint32_t at = 0xffffffffu;
        for (int b = block0; b < block1; ++b) {
            const float4 v = x4[b * 32 + lane];
            const uint32_t i = (uint32_t)(first + b * kBlock + lane * 4);
            if (v.w == m) at = min(at, i + 3);
            if (v.z == m) at = min(at, i + 2);
            if (v.y == m) at = min(at, i + 1);
            if (v.x == m) at = min(at, i);
        }
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) s.warp_word[warp] = at;
        __syncthreads();
        if (warp == 0) {
            at = __reduce_min_sync(0xffffffffu, lane < kSampleWarps ? s.warp_word[lane] : 0xffffffffu);
            if (lane < ranks) cluster.map_shared_rank(&s, lane)->rank_first[rank] = at;
        }
        all_here();
        if (rank == 0 && warp == 0) {
            at = __reduce_min_sync(0xffffffffu, lane < ranks ? s.rank_first[lane] : 0xffffffffu);
            if (lane == 0) {
                p.tokens[row] = (int32_t)at;
                if (p.log_probs) p.log_probs[row] = 0.f;
            }
        }
        return;
    }

    // Temperatures at which no number but the largest logit has a weight are all alike.
    const uint32_t m_key = key_of(m);
    const float below = fmaxf(value_of(m_key - 1), -FLT_MAX), t = fmaxf(temperature, (m - below) * (1.f / 256.f));
    Weigh weigh;
    weigh.c = 32. * 1.4426950408889634 / (double)t;
    weigh.mc = (double)m * weigh.c;
    weigh.floor = fmaxf(fminf(below, m - 44.3614f * t), -FLT_MAX);   // 64 ln 2
    const bool low = weigh.floor == -FLT_MAX;   // then minus infinity has to be told from the floor
    weigh.power = s.power;

    // ---- top-k and top-p: the lowest key that is kept whole, and how many logits of the key in front of it ----
    uint32_t keep = kLowestKey, tie_key = 0, ties = 0, tie_before = 0;   // (ties of the CTAs before this one)
    int pass = 0;
    // One pass: bins of the interval's logits, summed over the cluster; then the bin in which what lies above reaches the target.
    // want_total: every weight is added up too, and the target worked out from that.
    auto find = [&](const Interval& iv, uint64_t above_n, uint64_t above_w, bool by_weight, uint64_t& target, bool want_total) {
        const int buf = pass & 1;
        if (pass >= 2) {   // (its bins of two passes ago have been read: a barrier lies between)
            if (tid < kSampleBins) s.count[buf][tid] = s.low[buf][tid] = s.high[buf][tid] = 0;
            __syncthreads();
        }
        ++pass;
        uint64_t total = 0;
        for (int b = block0; b < block1; ++b) {
            const float4 v4 = x4[b * 32 + lane];
            const float v[4] = {v4.x, v4.y, v4.z, v4.w};
            uint64_t w[4];
            if (want_total) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = weigh(v[i]);
                    if (low && v[i] == -INFINITY) w[i] = 0;
                    total += w[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t key = key_of(v[i]);
                if (key < iv.lo || key > iv.hi) continue;
                const int at = iv.bin(v[i], key);
                const uint64_t u = want_total ? w[i] : weigh(v[i]);
                atomicAdd(&s.count[buf][at], 1u);
                const uint32_t lo = (uint32_t)u, old = atomicAdd(&s.low[buf][at], lo), hi = (uint32_t)(u >> 32) + (old + lo < old);
                if (hi) atomicAdd(&s.high[buf][at], hi);
            }
        }
        if (want_total) {
            total = warp_sum_u64(total);
            if (lane == 0) s.warp_sum[warp] = total;
            __syncthreads();
            if (warp == 0) {
                total = warp_sum_u64(lane < kSampleWarps ? s.warp_sum[lane] : 0);
                if (lane < ranks) cluster.map_shared_rank(&s, lane)->rank_total[rank] = total;
            }
        }
        all_here();
        if (tid < kSampleBins) {
            uint32_t n = 0, before = 0;
            uint64_t w = 0;
            for (int r = 0; r < ranks; ++r) {
                const SampleShared* from = cluster.map_shared_rank(&s, r);
                const uint32_t c = from->count[buf][tid];
                n += c;
                if (r < rank) before += c;
                w += ((uint64_t)from->high[buf][tid] << 32) + from->low[buf][tid];
            }
            s.number[tid] = n;
            s.before[tid] = before;
            s.weight[tid] = w;
        }
        if (want_total) {
            uint64_t all = 0;
            for (int r = 0; r < ranks; ++r) all += s.rank_total[r];
            target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), all, true));
        }
        __syncthreads();
        if (warp == 0) {   // lane l has bins 255 - 8 l down to 248 - 8 l
            uint64_t n = 0, w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n += s.number[kSampleBins - 1 - lane * 8 - i];
                w += s.weight[kSampleBins - 1 - lane * 8 - i];
            }
            const uint64_t n_to = above_n + warp_scan_u64(n, lane), w_to = above_w + warp_scan_u64(w, lane);
            const unsigned reached = __ballot_sync(0xffffffffu, (by_weight ? w_to : n_to) >= target);
            if (lane == (reached ? __ffs(reached) - 1 : 31)) {
                n = n_to - n;
                w = w_to - w;
                int at = kSampleBins - 1 - lane * 8;
                for (int i = 0; i < 8; ++i, --at) {
                    const uint64_t n1 = n + s.number[at], w1 = w + s.weight[at];
                    if ((by_weight ? w1 : n1) >= target) break;
                    n = n1;
                    w = w1;
                }
                if (!reached) at = -1;   // (n and w: everything)
                s.found.bin = at;
                s.found.above_n = (uint32_t)n;
                s.found.above_w = w;
                if (at >= 0) {
                    s.found.n = s.number[at];
                    s.found.w = s.weight[at];
                    s.found.before = s.before[at];
                }
            }
        }
        __syncthreads();
        return s.found;
    };
    // Keeps the front part that reaches `target` logits, or units, of those from key `bottom` on.
    // Returns the units of what lies above the ties, or is kept whole.
    auto select = [&](Interval iv, uint32_t bottom, bool by_weight, uint64_t target, bool want_total) {
        uint64_t above_n = 0, above_w = 0;
        const uint32_t old_ties = ties;
        for (;;) {
            const auto f = find(iv, above_n, above_w, by_weight, target, want_total);
            want_total = false;
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
                tie_before = f.before;
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
    uint64_t total_k = 0;
    if (by_count) {
        Interval iv;
        iv.by_key(max(kLowestKey, key_of(cut)), m_key);
        total_k = select(iv, kLowestKey, false, (uint64_t)top_k, false);
        if (ties > 0) total_k += ties * weigh(value_of(tie_key));
    }
    if (by_share) {
        const uint64_t target = max((uint64_t)1, share_of(fmaxf(top_p, 0.f), total_k, true));
        Interval iv;
        if (!by_count) {
            iv.by_key(max(kLowestKey, key_of(cut)), m_key);
            select(iv, kLowestKey, true, 0, true);
        } else if (keep <= m_key) {
            iv.by_key(keep, m_key);
            select(iv, keep, true, target, false);
        } else {   // all of what is left are equal
            const uint64_t w = weigh(value_of(tie_key));
            ties = (uint32_t)min((uint64_t)ties, (target + w - 1) / w);
        }
    }

    // ---- the kept weights' sums ----
    const uint64_t least = min_p > 0.f ? (uint64_t)ceil((double)fminf(min_p, 1.f) * (double)weigh(m)) : 0;
    uint32_t tie_at = 0;   // ties in front of the warp's next block
    if (ties > 0) {
        uint32_t n = 0;
        for (int b = block0; b < block1; ++b) {
            const float4 v = x4[b * 32 + lane];
            n += (key_of(v.x) == tie_key) + (key_of(v.y) == tie_key) + (key_of(v.z) == tie_key) + (key_of(v.w) == tie_key);
        }
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) s.warp_word[warp] = n;
        __syncthreads();
        tie_at = tie_before;
        for (int w = 0; w < warp; ++w) tie_at += s.warp_word[w];
    }
    // units of four neighbouring logits of block b, none where they are not kept; `at`: ties so far, moved on
    auto kept_units = [&](int b, uint32_t& at, uint64_t (&w)[4]) {
        const float4 v4 = x4[b * 32 + lane];
        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
        bool in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i] = key_of(v[i]) >= keep;
        if (ties > 0) {
            unsigned of[4], any = 0;
            const unsigned lower = (1u << lane) - 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) any |= of[i] = __ballot_sync(0xffffffffu, key_of(v[i]) == tie_key);
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
    {
        uint32_t at = tie_at;
        for (int b = block0; b < block1; ++b) {
            uint64_t w[4];
            kept_units(b, at, w);
            sum += (w[0] + w[1]) + (w[2] + w[3]);
        }
    }
    sum = warp_sum_u64(sum);
    if (lane == 0) s.warp_sum[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        const uint64_t all = warp_sum_u64(lane < kSampleWarps ? s.warp_sum[lane] : 0);
        if (lane < ranks) cluster.map_shared_rank(&s, lane)->rank_kept[rank] = all;
    }
    all_here();

    // ---- the draw ----
    uint64_t total = 0, in_front = 0;
    for (int r = 0; r < ranks; ++r) {
        total += s.rank_kept[r];
        if (r < rank) in_front += s.rank_kept[r];
    }
    for (int w = 0; w < warp; ++w) in_front += s.warp_sum[w];
    const float u = fmaxf(p.uniform[row], 0.f);
    const uint64_t drawn = u < 1.f ? share_of(u, total, false) : total - 1;   // the token's sum exceeds it
    if (drawn < in_front || drawn >= in_front + sum) return;
    for (int b = block0; b < block1; ++b) {
        uint64_t w[4];
        kept_units(b, tie_at, w);
        const uint64_t here = (w[0] + w[1]) + (w[2] + w[3]), to = in_front + warp_scan_u64(here, lane);
        const unsigned past = __ballot_sync(0xffffffffu, to > drawn);
        if (past) {
            if (lane == __ffs(past) - 1) {
                uint64_t at = to - here;
                int i = 0;
                for (; i < 3; ++i) {
                    at += w[i];
                    if (at > drawn) break;
                }
                const uint64_t units = i == 0 ? w[0] : i == 1 ? w[1] : i == 2 ? w[2] : w[3];
                p.tokens[row] = first + b * kBlock + lane * 4 + i;
                if (p.log_probs) p.log_probs[row] = (float)log((double)units / (double)total);
            }
            return;
        }
        in_front = __shfl_sync(0xffffffffu, to, 31);
    }
}

constexpr int kMaxStretch = (227 * 1024 - (int)sizeof(SampleShared)) / 4 / kBlock * kBlock;
static_assert((int64_t)kMaxStretch * kSampleRanks >= kMaxVocab + 8 + kSampleRanks * kBlock, "the largest vocabulary fits eight CTAs");

template <class F>
cudaError_t for_each_sample(F f) {
    cudaError_t e = f(sw_sample_kernel<float>);
    if (e == cudaSuccess) e = f(sw_sample_kernel<__nv_bfloat16>);
    if (e == cudaSuccess) e = f(sw_sample_kernel<__half>);
    return e;
}
cudaError_t configure_sample_kernels() {
    return for_each_sample([](auto* kernel) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SampleShared) + kMaxStretch * 4);
    });
}

cudaError_t launch_sample(const SampleParams& params, int dtype, int num_sms, cudaStream_t stream) {
    SampleParams p = params;
    // CTAs of a row: as many as give each 16384 logits at most (64 KB: two CTAs an SM, one loads while the other works), and more where rows are few.
    const int64_t positions = (int64_t)p.vocab + 16 / (dtype == SW_DTYPE_F32 ? 4 : 2) - 1;   // (a row may start anywhere behind a 16-byte boundary)
    int ranks = 1;
    while (ranks < kSampleRanks && (positions > ranks * 16384 || (p.rows * ranks < num_sms && positions > ranks * 2048))) ranks *= 2;
    p.stretch = (int)((positions + ranks * kBlock - 1) / (ranks * kBlock) * kBlock);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * ranks));
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = sizeof(SampleShared) + (size_t)p.stretch * 4;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return dtype == SW_DTYPE_F32    ? cudaLaunchKernelEx(&cfg, sw_sample_kernel<float>, p)
           : dtype == SW_DTYPE_BF16 ? cudaLaunchKernelEx(&cfg, sw_sample_kernel<__nv_bfloat16>, p)
                                    : cudaLaunchKernelEx(&cfg, sw_sample_kernel<__half>, p);
}

}  // namespace sw
