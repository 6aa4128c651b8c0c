// The mixed iteration inside a sliding window with sinks: the kernels of sw_mixed.cuh with kWindow.
//
// The row at position t attends key k when k <= t and (k > t - window or k < sinks).  Pages that hold no such key are passed over when the work
// is laid out: a decode request's visible pages are numbered without gaps (span_of), and the 128-key tiles of a chunk's item are made of the pages that
// its rows attend (pf_passed), so plan, line and pieces see only what is read.  In the pages at the window's edges the scores of unattended
// keys are masked.
#include "sw_mixed.cuh"

namespace sw {

cudaError_t configure_window_kernels(int head_dim) { return configure_option<kWindow>(head_dim); }
cudaError_t window_attn_resident_ctas_per_sm(int head_dim, int* out) { return resident_ctas_of_option<kWindow>(head_dim, out); }
cudaError_t launch_window_attn(int head_dim, const KvMaps& kv_maps, const CUtensorMap& q_map, const CUtensorMap& out_map, const MixedParams& p,
                               int num_sms, cudaStream_t stream) {
    return launch_option<kWindow>(head_dim, kv_maps, q_map, out_map, p, num_sms, stream);
}

}  // namespace sw
