// Eviction from the KV cache by accumulated weight: which keys of every (request, KV head) pair stay, then the copy of their rows.
//
// Of a pair's `len` keys the first `sinks` and the last `recent` stay, and of those between them the budget - sinks - recent heaviest (of equal
// weights the ones at the lowest positions; NaN counts as the lightest).  The kept keys keep their order.  They go to other pages and
// another row of weights: pages that requests share stay as they are, and no thread reads what another one writes.
//
// Selection (sw_evict_select_kernel): a cluster of 1 to 8 CTAs per pair finds the threshold by radix, 11 + 11 + 10 bits of the weights as ordered
// integers, with histograms in shared memory that the cluster's CTAs read from one another.  Each CTA has an equal stretch of the pair's keys, the
// first kHeldKeys of it in shared memory, so the weights are read from memory once.  A last pass writes the kept positions in order.
// Copy (sw_evict_move_kernel): one warp per (request, new page, KV head); bound by memory.
#include <cooperative_groups.h>

#include "sw_mixed.cuh"

namespace sw {
namespace cg = cooperative_groups;

constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 2048, kHeldKeys = 12288;   // 48 KB of keys: four CTAs on an SM
constexpr int kMoveThreads = 256;

struct SelectShared {
    uint32_t hist[kBins];
    uint32_t held[kHeldKeys];
    uint32_t scan[2][kSelectWarps];   // by the parity of the use
    uint32_t counts[2];   // keys above the threshold and at it in this CTA's stretch
    uint32_t digit, rest;
};

// Floats as integers of the same order; NaN as the lowest.
__device__ __forceinline__ uint32_t ordered(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);   // -0 as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Block-wide exclusive prefix sum of one value per thread; `total` is the block's.  `use` counts the calls: two in a row have different words, and
// every call has a barrier, so the words of the call before last are free.
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, SelectShared& s, int& use, uint32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    uint32_t* words = s.scan[use++ & 1];
    if (lane == 31) words[warp] = inc;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSelectWarps; ++w) {
        const uint32_t t = words[w];
        all += t;
        if (w < warp) before += t;
    }
    *total = all;
    return before + inc - v;
}

__global__ void __launch_bounds__(kSelectThreads) sw_evict_select_kernel(const EvictParams p) {
    extern __shared__ __align__(16) unsigned char select_raw[];
    SelectShared& s = *reinterpret_cast<SelectShared*>(select_raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int pair = blockIdx.x / ranks, i = pair / p.Hkv, h = pair % p.Hkv;
    for (int b = threadIdx.x; b < kBins; b += kSelectThreads) s.hist[b] = 0;
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
    const float* w = p.weights + ((int64_t)row * p.Hkv + h) * p.capacity;
    float* new_w = p.weights + ((int64_t)new_row * p.Hkv + h) * p.capacity;
    int32_t* list = p.kept + ((int64_t)i * p.Hkv + h) * p.budget;
    const int everything = rank * kSelectThreads + threadIdx.x, step = ranks * kSelectThreads;
    if (len <= p.budget) {
        for (int k = everything; k < len; k += step) {
            list[k] = k;
            new_w[k] = w[k];
        }
        return;
    }
    // the keys that stay without asking
    const int fixed = p.sinks + p.recent, wanted = p.budget - fixed;
    for (int k = everything; k < fixed; k += step) {
        const int slot = k < p.sinks ? k : p.budget - fixed + k, from = k < p.sinks ? k : len - fixed + k;
        list[slot] = from;
        new_w[slot] = w[from];
    }
    if (wanted == 0) return;
    const int keys = len - fixed;   // the others: positions sinks .. sinks + keys - 1
    const int begin = (int)((int64_t)keys * rank / ranks), mine = (int)((int64_t)keys * (rank + 1) / ranks) - begin;
    w += p.sinks + begin;
    const int held = min(mine, kHeldKeys);
    auto key_of = [&](int k) { return k < held ? s.held[k] : ordered(__ldg(w + k)); };

    uint32_t prefix = 0, rest = (uint32_t)wanted;   // bits of the threshold found so far; how many keys to take among those that share them
    int use = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : 2048;
        const uint32_t known = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);   // the bits that are fixed already
        if (pass > 0)
            for (int b = threadIdx.x; b < kBins; b += kSelectThreads) s.hist[b] = 0;
        __syncthreads();
        if (pass == 0) {
#pragma unroll 4
            for (int k = threadIdx.x; k < mine; k += kSelectThreads) {
                const uint32_t key = ordered(__ldg(w + k));
                if (k < held) s.held[k] = key;
                atomicAdd(&s.hist[key >> 21], 1u);
            }
        } else {
            for (int k = threadIdx.x; k < mine; k += kSelectThreads) {
                const uint32_t key = key_of(k);
                if ((key & known) == prefix) atomicAdd(&s.hist[(key >> shift) & (bins - 1)], 1u);
            }
        }
        cluster.sync();
        // four neighbouring bins per thread, from the highest down, summed over the cluster
        uint32_t n[4] = {0, 0, 0, 0}, all = 0, total;
        const int top = kBins - 1 - 4 * (int)threadIdx.x;
        for (int r = 0; r < ranks; ++r) {
            const uint4 v = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(s.hist, r) + top - 3);
            n[0] += v.w, n[1] += v.z, n[2] += v.y, n[3] += v.x;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) all += n[b];
        uint32_t before = block_prefix(all, s, use, &total);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (before < rest && before + n[b] >= rest) {   // exactly one thread and bin
                s.digit = (uint32_t)(top - b);
                s.rest = rest - before;
            }
            before += n[b];
        }
        cluster.sync();   // (also: nobody clears a histogram that another CTA still reads)
        prefix |= s.digit << shift;
        rest = s.rest;
        __syncthreads();
    }
    // keys above the threshold, and at it: of those the first `rest` by position
    uint32_t above = 0, equal = 0;
    for (int k = threadIdx.x; k < mine; k += kSelectThreads) {
        const uint32_t key = key_of(k);
        above += key > prefix;
        equal += key == prefix;
    }
    uint32_t total_above, total_equal;
    block_prefix(above, s, use, &total_above);
    block_prefix(equal, s, use, &total_equal);
    if (threadIdx.x == 0) {
        s.counts[0] = total_above;
        s.counts[1] = total_equal;
    }
    cluster.sync();
    uint32_t above_before = 0, equal_before = 0;
    for (int r = 0; r < rank; ++r) {
        const uint32_t* c = cluster.map_shared_rank(s.counts, r);
        above_before += c[0];
        equal_before += c[1];
    }
#pragma unroll 1
    for (int k0 = 0; k0 < mine; k0 += kSelectThreads) {
        const int k = k0 + threadIdx.x;
        const uint32_t key = k < mine ? key_of(k) : 0u;
        const bool is_above = k < mine && key > prefix, is_equal = k < mine && key == prefix;
        uint32_t tile;   // two counts of at most 512
        const uint32_t b = block_prefix((is_above ? 1u << 16 : 0u) | (is_equal ? 1u : 0u), s, use, &tile);
        const uint32_t my_above = above_before + (b >> 16), my_equal = equal_before + (b & 0xffffu);
        if (is_above || (is_equal && my_equal < rest)) {
            const int slot = p.sinks + (int)(my_above + min(my_equal, rest)), from = p.sinks + begin + k;
            list[slot] = from;
            new_w[slot] = w[k];
        }
        above_before += tile >> 16;
        equal_before += tile & 0xffffu;
    }
    cluster.sync();   // a CTA's counts and histogram are read by the others
}

// Lane groups of D / 8 lanes copy a row each, 16 bytes a lane; all loads of a page's K and V rows are in flight before the first store.
template <int D>
__global__ void __launch_bounds__(kMoveThreads) sw_evict_move_kernel(const EvictParams p) {
    constexpr int kRowLanes = D / 8, kRows = 32 / kRowLanes, kLoads = kPageSize / kRows;
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, sub = lane / kRowLanes, col = lane % kRowLanes * 8;
    const int new_pages = (p.budget - 1) / kPageSize + 1;
    const int64_t tasks = (int64_t)p.n * new_pages * p.Hkv;
    for (int64_t t = (int64_t)blockIdx.x * (kMoveThreads / 32) + threadIdx.x / 32; t < tasks; t += (int64_t)gridDim.x * (kMoveThreads / 32)) {
        const int h = (int)(t % p.Hkv), pg = (int)(t / p.Hkv % new_pages), i = (int)(t / p.Hkv / new_pages);
        const int rows = min(p.new_len[i] - pg * kPageSize, kPageSize);
        if (rows <= 0) continue;
        const int to = p.new_pages[p.new_page_indptr[i] + pg];
        int from = -1, page = -1;   // lane l < rows: position of slot l's row, and its page
        if (lane < rows) {
            from = p.kept[((int64_t)i * p.Hkv + h) * p.budget + pg * kPageSize + lane];
            page = p.pages[p.page_indptr[i] + from / kPageSize];
        }
        const bool bad = to < 0 || (int64_t)to >= p.num_pages || (lane < rows && (page < 0 || (int64_t)page >= p.num_pages));
        if (__any_sync(0xffffffffu, bad)) {
            if (lane == 0) report(p.ctrl, SW_ERR_OUT_OF_RANGE, kSiteEvict, i);
            continue;
        }
        uint4 k[kLoads], v[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int slot = j * kRows + sub;
            const int f = __shfl_sync(0xffffffffu, from, slot), pgid = __shfl_sync(0xffffffffu, page, slot);
            if (slot < rows) {
                const __nv_bfloat16* src = p.pool + ((((int64_t)pgid * 2 * p.Hkv) + h) * kPageSize + f % kPageSize) * D + col;
                k[j] = __ldcs(reinterpret_cast<const uint4*>(src));
                v[j] = __ldcs(reinterpret_cast<const uint4*>(src + (int64_t)p.Hkv * kPageSize * D));
            }
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int slot = j * kRows + sub;
            if (slot < rows) {
                __nv_bfloat16* dst = p.pool + ((((int64_t)to * 2 * p.Hkv) + h) * kPageSize + slot) * D + col;
                __stcs(reinterpret_cast<uint4*>(dst), k[j]);
                __stcs(reinterpret_cast<uint4*>(dst + (int64_t)p.Hkv * kPageSize * D), v[j]);
            }
        }
    }
}

cudaError_t configure_evict_kernels() {
    return cudaFuncSetAttribute(sw_evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SelectShared));
}

cudaError_t launch_evict(const EvictParams& p, int head_dim, int num_sms, cudaStream_t stream) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    // as many CTAs per pair as keep the launch within three CTAs an SM
    const int64_t pairs = (int64_t)p.n * p.Hkv;
    int ranks = 8;
    while (ranks > 1 && pairs * ranks > 3 * (int64_t)num_sms) ranks /= 2;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * ranks));
    cfg.blockDim = dim3(kSelectThreads);
    cfg.dynamicSmemBytes = sizeof(SelectShared);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, sw_evict_select_kernel, p);
    if (e != cudaSuccess) return e;
    const int64_t tasks = pairs * ((p.budget - 1) / kPageSize + 1), blocks = (tasks + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    cfg.gridDim = dim3((unsigned)(blocks < 8 * (int64_t)num_sms ? blocks : 8 * (int64_t)num_sms));
    cfg.blockDim = dim3(kMoveThreads);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    return head_dim == 64 ? cudaLaunchKernelEx(&cfg, sw_evict_move_kernel<64>, p) : cudaLaunchKernelEx(&cfg, sw_evict_move_kernel<128>, p);
}

}  // namespace sw
