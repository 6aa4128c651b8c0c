// Rotary positions: the iteration's queries and new keys turned by their positions, the keys written to their pages with their values (or to a tensor).
//
// Pair (a, b) of a head becomes (a cos - b sin, b cos + a sin) of its angle, position times the pair's frequency.  Far positions times fp32
// frequencies are off by whole turns' parts (131072 positions: 0.008 radians), so the frequencies are turns per position in 64 bits.  Their product
// with the position is off by 2^-53 of itself for its rounding and as much for the frequency's (the nearest integer is taken off without any): less than 2^-37 of a turn
// up to position 2^17, 2^-23 at 2^31 - 1.  Only what is left of a turn goes to 32 bits, with the sine and cosine of it.
//
// A lane holds 16 elements of a head, both elements of its eight pairs: two 16-byte pieces `rotary / 16` pieces apart, in either layout.  Lanes
// past the rotated part hold the rest.  4 (head size 128) or 8 heads lie side by side in a warp, so a lane's angles are the same for all heads of a row
// and worked out once per warp.  Bound by memory, or for few rows by its chain of latencies (length, page id, row, store).
// Measured, 32/8/128 with the append, launches in a graph: one row 2.4 us, 64 decodes 3.0, these beside a chunk of 512 5.2, 8192 rows 38.5 (201 MB at
// 81 % of a copy's rate).
#include "sw_mixed.cuh"

namespace sw {

// kRopeAhead: warp-wide parts of a row that are loaded at once.  (3 or 4 of them, 3 or 5 blocks an SM, the next part's loads in front of the last one's
// stores and loads marked as read once were tried for the 8192 rows, and none was faster.)
constexpr int kRopeThreads = 256, kRopeBlocksPerSm = 4, kRopeAhead = 2;

template <int D, bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads, kRopeBlocksPerSm) sw_rope_kernel(const RopeParams p) {
    constexpr int kLanes = D / 16, kHeads = 32 / kLanes;   // lanes of a head, heads side by side
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const int apart = p.rotary / 16;   // pieces between the two of a lane
    const bool turns = l < apart;
    const int piece_a = turns ? l : 2 * l, piece_b = turns ? l + apart : 2 * l + 1;
    const AppendParams& a = p.append;
    const int heads = p.Hq + a.Hkv * (a.pool ? 2 : 1);
    const int units = (a.C + a.n) * p.parts, stride = (int)(gridDim.x * (kRopeThreads / 32));
#pragma unroll 1
    for (int u = (int)(blockIdx.x * (kRopeThreads / 32) + threadIdx.x / 32); u < units; u += stride) {
        const int row = u / p.parts, part = u - row * p.parts;
        int h0 = part * p.part_heads;
        const int h_end = min(heads, h0 + p.part_heads);
        uint4 x[kRopeAhead][2];
        auto load = [&] {
#pragma unroll
            for (int b = 0; b < kRopeAhead; ++b) {
                const int h = h0 + b * kHeads + sub;
                if (h >= h_end) continue;
                const __nv_bfloat16* src = h < p.Hq ? p.q + row * p.q_stride + h * D
                                           : h < p.Hq + a.Hkv ? a.k_new + row * p.k_stride + (h - p.Hq) * D
                                                              : a.v_new + row * p.v_stride + (h - p.Hq - a.Hkv) * D;
                x[b][0] = *reinterpret_cast<const uint4*>(src + piece_a * 8);
                x[b][1] = *reinterpret_cast<const uint4*>(src + piece_b * 8);
            }
        };
        load();
        // the row's place in its sequence, and of its K and V in the pool (slot: -1 = nowhere)
        int pos, slot = -1;
        int64_t page = 0;
        {
            const int32_t* pages;
            int npages;
            if (row < a.C) {
                int cP = a.cP[0], cRow0 = 0, page0 = 0, page1 = a.cPage0[1];
#pragma unroll
                for (int j = 1; j < kMaxChunks; ++j)
                    if (j < a.nchunks && row >= a.cRow0[j]) {
                        cP = a.cP[j];
                        cRow0 = a.cRow0[j];
                        page0 = a.cPage0[j];
                        page1 = a.cPage0[j + 1];
                    }
                pos = (int)((unsigned)cP + (unsigned)(row - cRow0));
                pages = a.prefill_pages + page0;
                npages = page1 - page0;
            } else {
                const int i = row - a.C;
                pos = a.decode_kv_len[i] - 1;
                const int beg = a.decode_page_indptr[i];
                pages = a.decode_pages + beg;
                npages = a.decode_page_indptr[i + 1] - beg;
            }
            if (a.pool && h_end > p.Hq) {
                const unsigned at = (unsigned)pos / kPageSize;   // (a position of -1 lies in no list)
                if (at < (unsigned)max(npages, 0)) {
                    page = pages[at];
                    if (page < 0 || page >= a.num_pages) {
                        if (lane == 0) report(a.ctrl, SW_ERR_OUT_OF_RANGE, kSiteAppendPage, row);
                    } else {
                        slot = pos % kPageSize;
                    }
                } else if (lane == 0) {
                    report(a.ctrl, SW_ERR_OUT_OF_RANGE, kSiteAppendLen, row);
                }
            }
        }
        if (p.positions) pos = p.positions[row];
        float c[8], s[8];
        if (turns && h0 < p.Hq + a.Hkv) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int pair = !kInterleaved ? l * 8 + e : (e < 4 ? piece_a * 4 + e : piece_b * 4 + e - 4);
                double t = (double)pos * p.turns[pair];
                t -= rint(t);
                sincospif(2.f * (float)t, &s[e], &c[e]);
                s[e] *= p.magnitude;
                c[e] *= p.magnitude;
            }
        }
#pragma unroll 1
        for (;;) {
#pragma unroll
            for (int b = 0; b < kRopeAhead; ++b) {
                const int h = h0 + b * kHeads + sub;
                if (h >= h_end) continue;
                uint32_t w[8] = {x[b][0].x, x[b][0].y, x[b][0].z, x[b][0].w, x[b][1].x, x[b][1].y, x[b][1].z, x[b][1].w};
                if (turns && h < p.Hq + a.Hkv) {
                    float f[16];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        f[2 * i] = __uint_as_float(w[i] << 16);
                        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float& first = f[kInterleaved ? 2 * e : e];
                        float& second = f[kInterleaved ? 2 * e + 1 : e + 8];
                        const float y = first * c[e] - second * s[e];
                        second = second * c[e] + first * s[e];
                        first = y;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
                }
                __nv_bfloat16* dst;
                if (h < p.Hq) {
                    dst = p.q_out + ((int64_t)row * p.Hq + h) * D;
                } else if (!a.pool) {
                    dst = p.k_out + ((int64_t)row * a.Hkv + h - p.Hq) * D;
                } else {
                    if (slot < 0) continue;
                    const int side = h >= p.Hq + a.Hkv, head = h - p.Hq - side * a.Hkv;
                    dst = a.pool + (((page * 2 + side) * a.Hkv + head) * kPageSize + slot) * D;
                }
                *reinterpret_cast<uint4*>(dst + piece_a * 8) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(dst + piece_b * 8) = make_uint4(w[4], w[5], w[6], w[7]);
            }
            h0 += kRopeAhead * kHeads;
            if (h0 >= h_end) break;
            load();
        }
    }
}

cudaError_t launch_rope(const RopeParams& params, int head_dim, int num_sms, cudaStream_t stream) {
    RopeParams p = params;
    const int side_by_side = 32 / (head_dim / 16), heads = p.Hq + p.append.Hkv * (p.append.pool ? 2 : 1);
    const int64_t rows = p.append.C + p.append.n, warps = (int64_t)num_sms * kRopeBlocksPerSm * (kRopeThreads / 32);
    const int per_row = (heads + side_by_side - 1) / side_by_side;   // warp-wide parts of a row
    if (rows == 0) return cudaSuccess;
    // A warp takes as many parts of a row as leave work for every warp that the device holds: the angles are worked out once for all of them.
    const int64_t each = (rows * per_row + warps - 1) / warps;
    const int at_once = (int)(each < per_row ? each : per_row);
    p.parts = (per_row + at_once - 1) / at_once;
    p.part_heads = at_once * side_by_side;
    const int64_t blocks = (rows * p.parts + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks < num_sms * kRopeBlocksPerSm ? blocks : num_sms * kRopeBlocksPerSm));
    cfg.blockDim = dim3(kRopeThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (head_dim == 64) return cudaLaunchKernelEx(&cfg, p.interleaved ? sw_rope_kernel<64, true> : sw_rope_kernel<64, false>, p);
    return cudaLaunchKernelEx(&cfg, p.interleaved ? sw_rope_kernel<128, true> : sw_rope_kernel<128, false>, p);
}

}  // namespace sw
