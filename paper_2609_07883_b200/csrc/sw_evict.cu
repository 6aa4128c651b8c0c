// Eviction from the KV cache by accumulated weight: which keys of every (request, KV head) pair stay, then the copy of their rows.
//
// Of a pair's `len` keys the first `sinks` and the last `recent` stay, and of those between them the budget - sinks - recent heaviest (of equal
// weights the ones at the lowest positions; NaN counts as the lightest).  The kept keys keep their order.  They go to other pages and
// another row of weights: pages that requests share stay as they are, and no thread reads what another one writes.
//
// Selection (sw_evict_select_kernel): a cluster of 1 to 8 CTAs per pair finds the threshold by radix, digits of 8 bits of the weights as ordered
// integers: four at most, and none after one whose keys all stay.  Each CTA has an equal stretch of the pair's keys, the first ones of it in shared memory, so the weights are read from memory once, and a
// histogram per digit that the cluster's CTAs read from one another.  That traffic is what a pass costs beside its barrier: with digits of 11
// bits (three passes, 64 KB into every CTA of a cluster of eight) a 32768-token context took 22 us.  From the same histograms every CTA
// knows how many keys the CTAs before it keep, so a last round writes the kept positions in order.
// Copy: one warp per (request, new page, KV head); bound by memory.  The selecting CTAs do it themselves where they fill the SMs or have little to copy,
// a launch of its own (sw_evict_move_kernel) otherwise.
#include <cooperative_groups.h>

#include <algorithm>

#include "sw_mixed.cuh"

namespace sw {
namespace cg = cooperative_groups;

constexpr int kManyThreads = 512, kFewThreads = 256;   // of a selecting CTA
constexpr int kBins = 256, kHeldKeys = 16384, kMaxRanks = 8, kLoadsAhead = 8;
constexpr int kMoveThreads = 256;

struct SelectShared {
    uint32_t hist[2][kBins];          // keys of each digit, by the parity of the pass (eight words a digit, by lane: no faster)
    alignas(16) uint32_t all[kBins], before[kBins];   // summed over the cluster; over the CTAs before this one
    uint32_t above[kManyThreads / 32], equal[kManyThreads / 32];
    alignas(16) uint32_t found[4];                // the digit, keys above it in the cluster and in the CTAs before, keys of it in those
    alignas(16) uint32_t held[];                  // ordered()
};

// Floats as integers of the same order; NaN as the lowest.
__device__ __forceinline__ uint32_t ordered(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);   // -0 as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The rows of one new page of a pair that keeps `kept` keys (list: p.kept).  Lane groups of D / 8 lanes copy a row each, 16 bytes a lane; all loads of
// the page's K rows (then V's) are in flight before the first store.
template <int D>
__device__ __forceinline__ void move_page(const EvictParams& p, int i, int h, int pg, int kept) {
    constexpr int kRowLanes = D / 8, kRows = 32 / kRowLanes, kLoads = kPageSize / kRows;
    const int lane = threadIdx.x & 31, sub = lane / kRowLanes, col = lane % kRowLanes * 8;
    const int rows = min(kept - pg * kPageSize, kPageSize);
    if (rows <= 0) return;
    const int to = p.new_pages[p.new_page_indptr[i] + pg];
    int from = -1, page = -1;   // lane l < rows: position of slot l's row, and its page
    if (lane < rows) {
        from = __ldcg(p.kept + ((int64_t)i * p.Hkv + h) * p.budget + pg * kPageSize + lane);
        page = p.pages[p.page_indptr[i] + from / kPageSize];
    }
    const bool bad = to < 0 || (int64_t)to >= p.num_pages || (lane < rows && (page < 0 || (int64_t)page >= p.num_pages));
    if (__any_sync(0xffffffffu, bad)) {
        if (lane == 0) report(p.ctrl, SW_ERR_OUT_OF_RANGE, kSiteEvict, i);
        return;
    }
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const __nv_bfloat16* src = p.pool + (int64_t)side * p.Hkv * kPageSize * D + col;
        __nv_bfloat16* dst = p.pool + (((int64_t)to * 2 + side) * p.Hkv + h) * kPageSize * D + col;
        uint4 x[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int slot = j * kRows + sub;
            const int f = __shfl_sync(0xffffffffu, from, slot), id = __shfl_sync(0xffffffffu, page, slot);
            if (slot < rows) x[j] = __ldcs(reinterpret_cast<const uint4*>(src + (((int64_t)id * 2 * p.Hkv + h) * kPageSize + f % kPageSize) * D));
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (j * kRows + sub < rows) __stcs(reinterpret_cast<uint4*>(dst + (j * kRows + sub) * D), x[j]);
    }
}

// D: head size where the cluster copies its pair's rows as well, 0 where a launch of its own does.
template <int D, int kSelectThreads>
__global__ void __launch_bounds__(kSelectThreads, 1024 / kSelectThreads) sw_evict_select_kernel(const EvictParams p) {
    constexpr int kSelectWarps = kSelectThreads / 32;
    extern __shared__ __align__(16) unsigned char select_raw[];
    SelectShared& s = *reinterpret_cast<SelectShared*>(select_raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int pair = blockIdx.x / ranks, i = pair / p.Hkv, h = pair % p.Hkv;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    static_assert(kSelectThreads >= kBins, "a thread per bin");
    if (threadIdx.x < kBins) s.hist[0][threadIdx.x] = s.hist[1][threadIdx.x] = 0;
    grid_launch_dependents();
    grid_dependency_wait();

    // (the same for all CTAs of the cluster)
    const int len = p.kv_len[i], row = p.row_of[i], new_row = p.new_row_of[i];
    const int pages = len > 0 ? (len - 1) / kPageSize + 1 : 0, kept = min(max(len, 0), p.budget);
    const int listed = p.page_indptr[i + 1] - p.page_indptr[i], new_listed = p.new_page_indptr[i + 1] - p.new_page_indptr[i];
    const bool fits = pages <= listed && (kept + kPageSize - 1) / kPageSize <= new_listed && len <= p.capacity &&
                      row >= 0 && (int64_t)row < p.rows && new_row >= 0 && (int64_t)new_row < p.rows && row != new_row;
    if (rank == 0 && h == 0 && threadIdx.x == 0) {
        p.new_len[i] = fits ? kept : 0;
        if (!fits) report(p.ctrl, SW_ERR_OUT_OF_RANGE, kSiteEvict, i);
    }
    if (!fits || kept == 0) return;
    auto all_here = [&] {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };
    auto move = [&](int count, bool listed_already = false) {   // (in step with the cluster's other CTAs, which write parts of the list)
        if constexpr (D > 0) {
            if (!listed_already) all_here();
            for (int pg = rank * kSelectWarps + warp; pg * kPageSize < count; pg += ranks * kSelectWarps) move_page<D>(p, i, h, pg, count);
        }
    };
    const float* w = p.weights + ((int64_t)row * p.Hkv + h) * p.capacity;
    float* new_w = p.weights + ((int64_t)new_row * p.Hkv + h) * p.capacity;
    int32_t* list = p.kept + ((int64_t)i * p.Hkv + h) * p.budget;
    const int everything = rank * kSelectThreads + threadIdx.x, step = ranks * kSelectThreads;
    if (len <= p.budget) {
        for (int k = everything; k < len; k += step) {
            list[k] = k;
            new_w[k] = w[k];
        }
        move(kept);
        return;
    }
    const int fixed = p.sinks + p.recent, wanted = p.budget - fixed;
    const int keys = len - fixed;   // those that are asked: positions sinks .. sinks + keys - 1
    const int begin = (int)((int64_t)keys * rank / ranks), mine = (int)((int64_t)keys * (rank + 1) / ranks) - begin;
    const float* x0 = w + p.sinks + begin;
    const int held = min(mine, p.held);
    // four neighbours from k on (a multiple of four), zeros past the end
    auto keys_of = [&](int k, uint32_t (&x)[4]) {
        if (k + 4 <= held) {
            const uint4 v = *reinterpret_cast<const uint4*>(s.held + k);
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = k + u >= mine ? 0u : (k + u < held ? s.held[k + u] : ordered(__ldg(x0 + k + u)));
        }
    };

    uint32_t prefix = 0, rest = (uint32_t)wanted;   // digits of the threshold so far; how many keys to take among those that share them
    uint32_t above_before = 0, equal_before = 0;    // keys above the threshold, and at it, in the CTAs before this one
    __syncthreads();
#pragma unroll 1
    for (int pass = 0; wanted > 0 && pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        uint32_t* hist = s.hist[pass & 1];
        if (pass == 0) {
            for (int k0 = threadIdx.x; k0 < mine; k0 += kLoadsAhead * kSelectThreads) {
                float x[kLoadsAhead];
#pragma unroll
                for (int u = 0; u < kLoadsAhead; ++u) x[u] = k0 + u * kSelectThreads < mine ? __ldg(x0 + k0 + u * kSelectThreads) : 0.f;
#pragma unroll
                for (int u = 0; u < kLoadsAhead; ++u) {
                    const int k = k0 + u * kSelectThreads;
                    if (k < mine) {
                        const uint32_t key = ordered(x[u]);
                        if (k < held) s.held[k] = key;
                        atomicAdd(&hist[key >> 24], 1u);
                    }
                }
            }
        } else {
#pragma unroll 2
            for (int k = 4 * threadIdx.x; k < mine; k += 4 * kSelectThreads) {
                uint32_t x[4];
                keys_of(k, x);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (k + u < mine && x[u] - prefix < 256u << shift) atomicAdd(&hist[x[u] >> shift & (kBins - 1)], 1u);
            }
        }
        all_here();   // (also: nobody reads the histogram of the pass before any more)
        if (threadIdx.x < kBins) {
            uint32_t n[kMaxRanks], all = 0, before = 0;   // all in flight at once
#pragma unroll
            for (int r = 0; r < kMaxRanks; ++r) n[r] = r < ranks ? cluster.map_shared_rank(hist, r)[threadIdx.x] : 0u;
#pragma unroll
            for (int r = 0; r < kMaxRanks; ++r) {
                all += n[r];
                before += r < rank ? n[r] : 0u;
            }
            s.all[threadIdx.x] = all;
            s.before[threadIdx.x] = before;
            s.hist[~pass & 1][threadIdx.x] = 0;
        }
        __syncthreads();
        if (threadIdx.x < 32) {   // eight neighbouring bins a lane, from the highest down
            const int top = kBins - 8 * (lane + 1);
            const uint4 a0 = *reinterpret_cast<const uint4*>(s.all + top + 4), a1 = *reinterpret_cast<const uint4*>(s.all + top);
            const uint4 b0 = *reinterpret_cast<const uint4*>(s.before + top + 4), b1 = *reinterpret_cast<const uint4*>(s.before + top);
            const uint32_t n[8] = {a0.w, a0.z, a0.y, a0.x, a1.w, a1.z, a1.y, a1.x}, m[8] = {b0.w, b0.z, b0.y, b0.x, b1.w, b1.z, b1.y, b1.x};
            uint32_t all = 0, before = 0;
#pragma unroll
            for (int b = 0; b < 8; ++b) all += n[b], before += m[b];
            uint32_t n_sum = all, m_sum = before;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t a = __shfl_up_sync(0xffffffffu, n_sum, o), c = __shfl_up_sync(0xffffffffu, m_sum, o);
                if (lane >= o) n_sum += a, m_sum += c;
            }
            n_sum -= all;   // in the bins above the lane's
            m_sum -= before;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                if (n_sum < rest && n_sum + n[b] >= rest)   // exactly one bin of one lane
                    *reinterpret_cast<uint4*>(s.found) = make_uint4((uint32_t)(top + 7 - b) | (n_sum + n[b] == rest ? kBins : 0u), n_sum, m_sum, m[b]);
                n_sum += n[b];
                m_sum += m[b];
            }
        }
        __syncthreads();   // (also: the sums are read before they are written again)
        const uint4 found = *reinterpret_cast<const uint4*>(s.found);
        prefix |= (found.x & (kBins - 1)) << shift;
        rest -= found.y;
        above_before += found.z;
        equal_before = found.w;
        if (found.x >= kBins && prefix > 0) {   // all keys that share these digits stay: the threshold is the number below them.  For most weights two or three digits do.
            prefix -= 1;
            above_before += equal_before;
            rest = equal_before = 0;
            break;
        }
    }
    // the keys that stay without asking
    for (int k = everything; k < fixed; k += step) {
        const int slot = k < p.sinks ? k : p.budget - fixed + k, from = k < p.sinks ? k : len - fixed + k;
        list[slot] = from;
        new_w[slot] = w[from];
    }
    if (wanted == 0) {
        move(kept);
        return;
    }
    // Each warp lists the keys of a stretch of its own: it counts them, adds those of the warps before, and goes over them again in order of position.
    // (In one pass, with a prefix sum over the CTA per 2048 keys: 81 against 69 us for 224 contexts of 928 to 4230 tokens to 43 keys.)
    const int stretch = ((mine - 1) / (kSelectWarps * 128) + 1) * 128, end = min(mine, (warp + 1) * stretch);
    uint32_t above = 0, equal = 0;
    for (int k = warp * stretch + 4 * lane; k < end; k += 128) {
        uint32_t x[4];
        keys_of(k, x);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            above += k + u < mine && x[u] > prefix;
            equal += k + u < mine && x[u] == prefix;
        }
    }
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) s.above[warp] = above, s.equal[warp] = equal;
    __syncthreads();
    above_before += __reduce_add_sync(0xffffffffu, lane < warp ? s.above[lane] : 0u);
    equal_before += __reduce_add_sync(0xffffffffu, lane < warp ? s.equal[lane] : 0u);
#pragma unroll 1
    for (int k0 = warp * stretch; k0 < end; k0 += 128) {
        const int first = k0 + 4 * lane;
        uint32_t x[4], flags = 0, counts = 0;   // bit u: above, bit 4 + u: equal; two counts of at most 128
        keys_of(first, x);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (first + u < mine && x[u] > prefix) flags |= 1u << u, counts += 1u << 16;
            if (first + u < mine && x[u] == prefix) flags |= 16u << u, counts += 1u;
        }
        if (!__any_sync(0xffffffffu, flags)) continue;
        uint32_t sum = counts;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t c = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += c;
        }
        const uint32_t tile = __shfl_sync(0xffffffffu, sum, 31);
        uint32_t my_above = above_before + (sum - counts >> 16), my_equal = equal_before + (sum - counts & 0xffffu);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool is_above = flags >> u & 1, is_equal = flags >> (4 + u) & 1;
            if (is_above || (is_equal && my_equal < rest)) {
                const int slot = p.sinks + (int)(my_above + min(my_equal, rest));
                list[slot] = p.sinks + begin + first + u;
                // the weight itself where its key stands for several: NaN, zeros
                new_w[slot] = x[u] == 0u || x[u] == 0x80000000u ? __ldg(x0 + first + u) : __uint_as_float(x[u] & 0x80000000u ? x[u] ^ 0x80000000u : ~x[u]);
            }
            my_above += is_above;
            my_equal += is_equal;
        }
        above_before += tile >> 16;
        equal_before += tile & 0xffffu;
    }
    all_here();   // a CTA's last histogram is read by the others
    if constexpr (D > 0) move(kept, true);
}

// One launch: a warp per (request, new page, KV head).
template <int D>
__global__ void __launch_bounds__(kMoveThreads) sw_evict_move_kernel(const EvictParams p) {
    grid_dependency_wait();
    const int new_pages = (p.budget - 1) / kPageSize + 1;
    const int64_t tasks = (int64_t)p.n * new_pages * p.Hkv;
    for (int64_t t = (int64_t)blockIdx.x * (kMoveThreads / 32) + threadIdx.x / 32; t < tasks; t += (int64_t)gridDim.x * (kMoveThreads / 32)) {
        const int h = (int)(t % p.Hkv), pg = (int)(t / p.Hkv % new_pages), i = (int)(t / p.Hkv / new_pages);
        move_page<D>(p, i, h, pg, p.new_len[i]);
    }
}

template <class F>
cudaError_t for_each_select(F f) {
    for (auto* kernel : {sw_evict_select_kernel<0, kManyThreads>, sw_evict_select_kernel<64, kManyThreads>, sw_evict_select_kernel<128, kManyThreads>,
                         sw_evict_select_kernel<0, kFewThreads>, sw_evict_select_kernel<64, kFewThreads>, sw_evict_select_kernel<128, kFewThreads>})
        if (const cudaError_t e = f(kernel)) return e;
    return cudaSuccess;
}
cudaError_t configure_evict_kernels() {
    return for_each_select([](auto* kernel) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(SelectShared) + kHeldKeys * sizeof(float)));
    });
}

cudaError_t launch_evict(const EvictParams& params, int head_dim, int num_sms, cudaStream_t stream) {
    EvictParams p = params;
    const int64_t pairs = (int64_t)p.n * p.Hkv;
    // As many CTAs per pair as keep the launch within two CTAs an SM, and as hold the longest row of weights in shared memory (61 contexts of 40606 to 131072
    // tokens, 4 KV heads: 148 us with eight, 173 us with one).
    int ranks = kMaxRanks;
    while (ranks > 1 && pairs * ranks > 2 * (int64_t)num_sms && p.capacity <= ranks / 2 * kHeldKeys) ranks /= 2;
    p.held = std::min(kHeldKeys, (p.capacity - 1) / ranks + 1);
    // Smaller CTAs where there is little for each one to do.  Pairs for more than two large CTAs an SM: 128 contexts of 2048 to 4096 tokens to 64 keys, 8 KV heads,
    // 32 against 43 us; 64 of 8192 to 16384 to 1024, though, 183 against 124.  Fewer pairs: one context of 8192 to 1024 12.6 against 14.4, of 32768 to 8192 25.7 against 24.7.
    const bool few = p.capacity <= (pairs > 2 * (int64_t)num_sms ? 8192 : 1024 * ranks);
    const int threads = few ? kFewThreads : kManyThreads;
    // One launch where the selecting CTAs fill the SMs or have a page a warp at most to copy (2 contexts of 524 to 584 tokens to 18: 10.8 against 12.4 us; one
    // of 32768 to 8192, which has more, 32.7 against 24.4).
    const bool fused = pairs * ranks >= num_sms || (p.budget - 1) / kPageSize < ranks * (threads / 32);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * ranks));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = sizeof(SelectShared) + (size_t)p.held * sizeof(float);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    auto* select = few ? (!fused ? sw_evict_select_kernel<0, kFewThreads> : head_dim == 64 ? sw_evict_select_kernel<64, kFewThreads> : sw_evict_select_kernel<128, kFewThreads>)
                       : (!fused ? sw_evict_select_kernel<0, kManyThreads> : head_dim == 64 ? sw_evict_select_kernel<64, kManyThreads> : sw_evict_select_kernel<128, kManyThreads>);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, select, p);
    if (e != cudaSuccess || fused) return e;
    const int64_t tasks = pairs * ((p.budget - 1) / kPageSize + 1), blocks = (tasks + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    cfg.gridDim = dim3((unsigned)(blocks < 8 * (int64_t)num_sms ? blocks : 8 * (int64_t)num_sms));
    cfg.blockDim = dim3(kMoveThreads);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    return head_dim == 64 ? cudaLaunchKernelEx(&cfg, sw_evict_move_kernel<64>, p) : cudaLaunchKernelEx(&cfg, sw_evict_move_kernel<128>, p);
}

}  // namespace sw
