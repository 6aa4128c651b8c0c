// Decode attention that also adds up the weight every key gets: the kernels of sw_mixed.cuh with kScored, then one pass over their scores.
//
// The weight of key k for request i and a KV head is the sum over the head's group of exp(s - lse), and lse is only known once all of the
// request's keys are done.  The attention leaves its scores behind (4 bytes per key and query head beside the 4 * D bytes per key and KV
// head that it reads: 1/32 of the traffic with four heads of 128 in a group); this pass, from L2 for the most part, turns them into weights.  A
// second look at the keys instead would read half the cache again.
//
// Every (request, KV head, key) has one owner, so the sums do not depend on any order.
#include "sw_mixed.cuh"

namespace sw {

constexpr int kWeightThreads = 256, kWeightBlocksPerSm = 4;

// A warp has an equal stretch of the entries of decode_pages; of a page, lane l has key l % 16 and every second KV head.
//
// Scores that have been read are discarded from L2: written back to memory, as 25 MB of them are in the course of four contexts of 49152 tokens, they
// cost the launches 7 us of 147.
__global__ void __launch_bounds__(kWeightThreads, kWeightBlocksPerSm) sw_key_weights_kernel(const WeightParams p) {
    grid_launch_dependents();
    // The batch was there before the attention launch started: where the warp's stretch lies is found while that ends (64 contexts of 256-2048
    // tokens 68.4 -> 60.9 us; with the request's other words as well 63.4).
    const int lane = threadIdx.x & 31, warps = gridDim.x * (kWeightThreads / 32), w = blockIdx.x * (kWeightThreads / 32) + threadIdx.x / 32;
    const int first = __ldcg(p.page_indptr);   // (the batch may be the later requests of a longer list)
    const int64_t total = (int64_t)__ldcg(p.page_indptr + p.n) - first;
    const int begin = first + (int)(total * w / warps), end = first + (int)(total * (w + 1) / warps);
    int i = 0;
    for (int hi = p.n; hi - i > 1;) {   // largest i with page_indptr[i] <= begin
        const int mid = (i + hi) >> 1;
        if (__ldcg(p.page_indptr + mid) <= begin) i = mid; else hi = mid;
    }
    grid_dependency_wait();
    const int spoiled = ld_relaxed_gpu(&p.ctrl[kCtrSpoiled]);   // (looked at with the first request's words)
    constexpr float kLog2E = 1.4426950408889634f;
    const int key = lane & 15, g = p.group, lines = p.Hkv * kPageSize * g / 32;   // of 128 bytes, of a page's scores
    int at = 0, next = begin, len = 0, row = 0;
    bool ok = false;
    for (int e = begin; e < end; ++e) {
        if (e == begin || e >= next) {
            while (p.page_indptr[i + 1] <= e) ++i;
            at = p.page_indptr[i];
            next = p.page_indptr[i + 1];
            len = p.kv_len[i];
            row = p.row_of[i];
            const int pages = len > 0 ? (len - 1) / kPageSize + 1 : 0;
            ok = pages <= next - at && at <= e;   // (reported by the attention launch; offsets that decrease have no entry of theirs here)
            ok = ok && spoiled == 0;   // some scores may not have been written
            if (ok && len > 0 && (row < 0 || (int64_t)row >= p.rows || len > p.capacity)) {
                if (lane == 0) report(p.ctrl, SW_ERR_OUT_OF_RANGE, kSiteWeights, i);
                ok = false;
            }
        }
        const int pos = (e - at) * kPageSize + key;
        if (ok && pos - key < len && e >= p.score_pages) {
            if (lane == 0) report(p.ctrl, SW_ERR_WORKSPACE, kSiteScratch, e);
            ok = false;   // (like all pages behind it)
        }
        const float* scores = p.scores + (int64_t)e * p.Hkv * kPageSize * g;
        if (ok && pos < len) {
            const float* lse = p.lse + (int64_t)i * p.Hkv * g;
            float* dst = p.weights + (int64_t)row * p.Hkv * p.capacity + pos;
#pragma unroll 4
            for (int h = lane >> 4; h < p.Hkv; h += 2) {
                const float before = pos == len - 1 ? 0.f : dst[(int64_t)h * p.capacity];   // the key of this step starts at nothing
                const float* s0 = scores + (h * kPageSize + key) * g;
                float sum = 0.f;
                if (g == 4) {
                    const float4 s = __ldcs(reinterpret_cast<const float4*>(s0));
                    const float4 l = __ldg(reinterpret_cast<const float4*>(lse + h * 4));
                    sum = (fast_exp2(fmaf(l.x, -kLog2E, s.x)) + fast_exp2(fmaf(l.y, -kLog2E, s.y))) +
                          (fast_exp2(fmaf(l.z, -kLog2E, s.z)) + fast_exp2(fmaf(l.w, -kLog2E, s.w)));
                } else {
                    for (int r = 0; r < g; ++r) sum += fast_exp2(fmaf(__ldg(lse + h * g + r), -kLog2E, __ldcs(s0 + r)));
                }
                dst[(int64_t)h * p.capacity] = before + sum;
            }
        }
        __syncwarp();
        if (e < p.score_pages && (lines * 32) == p.Hkv * kPageSize * g)
            for (int l = lane; l < lines; l += 32) asm volatile("discard.global.L2 [%0], 128;" ::"l"(scores + l * 32) : "memory");
    }
}

cudaError_t configure_scored_kernels(int head_dim) { return configure_option<kScored>(head_dim); }
cudaError_t launch_scored_attn(int head_dim, const KvMaps& kv_maps, const CUtensorMap& any_map, const MixedParams& p, int num_sms, cudaStream_t stream) {
    return launch_option<kScored>(head_dim, kv_maps, any_map, any_map, p, num_sms, stream);
}
cudaError_t launch_key_weights(const WeightParams& p, int num_sms, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)num_sms * kWeightBlocksPerSm);
    cfg.blockDim = dim3(kWeightThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sw_key_weights_kernel, p);
}

}  // namespace sw
