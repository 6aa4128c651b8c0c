// Launches of the append and of the mixed iteration (kernels: sw_mixed.cuh).
#include "sw_mixed.cuh"

namespace sw {

constexpr int kAppendThreads = 256, kAppendBlocksPerSm = 4;
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocksPerSm) sw_kv_append_kernel(const AppendParams p) {
    // launched with programmatic stream serialization: it may start while the previous kernel (the attention of
    // the previous iteration, possibly still reading this pool) drains; nothing is touched before this wait
    grid_launch_dependents();
    grid_dependency_wait();
    append_rows<true, 1>(p, p.D, (int)(blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32), (int)(gridDim.x * (blockDim.x / 32)));
}

cudaError_t launch_kv_append(const AppendParams& p, int num_sms, cudaStream_t stream) {
    const int pieces_per_row = p.Hkv * p.D / 8, rows_at_once = pieces_per_row < 32 ? 32 / pieces_per_row : 1;
    const int64_t total = (int64_t)((p.C + p.n + rows_at_once - 1) / rows_at_once) * ((pieces_per_row + 31) / 32);   // warp-wide parts
    if (total == 0) return cudaSuccess;
    const int threads = kAppendThreads;
    int64_t blocks = (total + threads / 32 - 1) / (threads / 32);
    // The grid is resident at once, so that the launch after this one is released at once too.  (Four parts a warp and grids of eight
    // blocks per SM: 3000 rows of 32/8/128 5.5 us instead of 5.2, 8192 10.7 instead of 10.3.  Eight blocks of 32 registers are as
    // fast alone and 1 us slower with the attention launch behind them, 461 rows 20.2 instead of 19.3 us.)
    if (blocks > (int64_t)num_sms * kAppendBlocksPerSm) blocks = (int64_t)num_sms * kAppendBlocksPerSm;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sw_kv_append_kernel, p);
}

// Self-test of the bounded wait: one warp waits on a barrier that nothing will ever complete; the wait must give up
// after `budget_cycles`, record SW_ERR_DEVICE_TIMEOUT in the status word and let the kernel end normally.
__global__ void sw_selftest_wait_kernel(int32_t* ctrl, long long budget_cycles) {
    __shared__ __align__(8) unsigned long long bar;
    const uint32_t addr = smem_u32(&bar);
    if (threadIdx.x == 0) {
        mbar_init(addr, 1);
        fence_mbar_init();
    }
    __syncwarp();
    if (!mbar_wait(addr, 0, budget_cycles) && threadIdx.x == 0) report(ctrl, SW_ERR_DEVICE_TIMEOUT, kSiteWait, 0xABCD);
}

cudaError_t launch_selftest_wait(int32_t* ctrl, long long budget_cycles, cudaStream_t stream) {
    sw_selftest_wait_kernel<<<1, 32, 0, stream>>>(ctrl, budget_cycles);
    return cudaGetLastError();
}

cudaError_t configure_kernels(int head_dim) { return configure_option<kPlain>(head_dim); }

// CTAs of the persistent kernel that one SM can hold at a time (the smallest figure of all forms).  The fused launch
// makes CTAs wait for one another's share of the KV append, which is only safe when the whole grid is resident.
cudaError_t mixed_attn_resident_ctas_per_sm(int head_dim, int* out) { return resident_ctas_of_option<kPlain>(head_dim, out); }

cudaError_t launch_mixed_attn(int head_dim, const KvMaps& kv_maps, const CUtensorMap& q_map, const CUtensorMap& out_map,
                              const MixedParams& p, int num_sms, cudaStream_t stream) {
    return launch_option<kPlain>(head_dim, kv_maps, q_map, out_map, p, num_sms, stream);
}

}  // namespace sw
