// Cross attention over the cached states of an encoder: the kernels of sw_mixed.cuh with kCross.
//
// Every row of a chunk attends all keys of its page list, whatever their number and the chunk's, so all items of a chunk take the same number of
// steps and only the last key tile is masked.  A decode request's row attends its keys as always; rows of requests without keys are zeroed where the
// lengths are read.
// The arithmetic is the plain iteration's.  Softmax weights are rounded to bf16 where they meet V: both operands of a 16-bit matrix instruction have one type.  Their
// sum is kept in 32 bits.  Against 64 bits outputs are off by 1.9e-3 (single tokens) to 2.3e-3 (chunks) of themselves (2-norm), where weights of 32 bits leave the
// 1.7e-3 of the output's own rounding.  To be rid of the difference each weight would have to be split in two, and the second matrix product be done twice.
// Bound as the plain iteration is: single tokens by the cached bytes (64 of them over 1500 keys each of 16/16/64, 393 MB: 63.5 us, 96 % of a copy's rate), chunks by
// the softmax between two matrix products (2048 rows over 16384 keys of 32/8/128: 459 to 493 us by the machine, 66 to 70 % of the matrix
// rate).
#include "sw_mixed.cuh"

namespace sw {

cudaError_t configure_cross_kernels(int head_dim) { return configure_option<kCross>(head_dim); }
cudaError_t launch_cross_attn(int head_dim, const KvMaps& kv_maps, const CUtensorMap& q_map, const CUtensorMap& out_map, const MixedParams& p,
                              int num_sms, cudaStream_t stream) {
    return launch_option<kCross>(head_dim, kv_maps, q_map, out_map, p, num_sms, stream);
}

// Rows of chunks without keys (the host knows which): `pieces` 16-byte pieces of out to zero, log-sum-exps of minus infinity.
__global__ void sw_keyless_rows_kernel(uint4* out, int64_t pieces, float* lse, int64_t values) {
    const int64_t first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = first; i < pieces; i += stride) out[i] = make_uint4(0, 0, 0, 0);
    for (int64_t i = first; i < values; i += stride) lse[i] = -INFINITY;
}
cudaError_t launch_keyless_rows(__nv_bfloat16* out, int64_t elements, float* lse, int64_t values, int num_sms, cudaStream_t stream) {
    const int64_t blocks = (elements / 8 + 255) / 256;
    sw_keyless_rows_kernel<<<(unsigned)(blocks < 4 * num_sms ? blocks : 4 * num_sms), 256, 0, stream>>>(reinterpret_cast<uint4*>(out), elements / 8, lse,
                                                                                                        lse ? values : 0);
    return cudaGetLastError();
}

}  // namespace sw
