// The KV pool held in 8 bits: append, and the mixed iteration that reads it (kernels of sw_mixed.cuh with kKv8).
//
// Pool: e4m3 [num_pages][2 (K, V)][Hkv][16][D]; scales: fp32 [num_pages][2][Hkv], powers of two.  An element of a block (page, K|V, head)
// stands for its e4m3 value times the block's scale.  A power of two costs a floating-point format no precision, and it makes two things
// exact: every element is a bf16 number (the attention's products see exactly what the cache stands for), and a block whose scale has to
// grow for a later row only moves its older rows' exponents (rounded again only where they become subnormal).
#include "sw_mixed.cuh"

namespace sw {

constexpr int kMinScaleExp = -100;   // 2^-100: blocks of zeros, and of values below any use
constexpr int kKv8Threads = 256;

// The blocks that an append writes, numbered: the pages of chunk 0 that get rows, of chunk 1, ..., then one of each decode request.
struct Kv8Params {
    AppendParams a;
    int block0[kMaxChunks + 1];   // written (expand: the prompt's) pages before chunk j's
    int cC[kMaxChunks];
    uint8_t* pool;
    float* scales;
    __nv_bfloat16* copy;   // expand only
    int32_t* list;
};

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
// Four e4m3 values times `f`, back to e4m3.
__device__ __forceinline__ uint32_t rescale_e4m3x4(uint32_t w, float f) {
    const float2 x = f32x2_of_f16x2(f16x2_of_e4m3(w)), y = f32x2_of_f16x2(f16x2_of_e4m3(w >> 16));
    return e4m3x4_of(x.x * f, x.y * f, y.x * f, y.y * f);
}

// sw_kv8_append: one warp per block.  The block's new rows (up to 16 of D elements) are held in registers, 16 bytes per lane and row, while
// their largest magnitude is found; bf16 magnitudes compare as integers, infinities and NaN above all finite ones.  Bound by memory: 2 bytes
// read and 1 written an element, and a chain of dependent loads (length, list offset, page id, scale) beside the rows' own.
template <int D>
__global__ void __launch_bounds__(kKv8Threads) sw_kv8_append_kernel(const Kv8Params p) {
    constexpr int kRowLanes = D / 8, kRows = 32 / kRowLanes, kLoads = kPageSize / kRows;
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, sides = 2 * p.a.Hkv;
    const int sub = lane / kRowLanes, col = lane % kRowLanes * 8;
    const int64_t tasks = (int64_t)(p.block0[p.a.nchunks] + p.a.n) * sides;
    for (int64_t t = (int64_t)blockIdx.x * (kKv8Threads / 32) + threadIdx.x / 32; t < tasks; t += (int64_t)gridDim.x * (kKv8Threads / 32)) {
        const int b = (int)(t / sides), side = (int)(t % sides) / p.a.Hkv, kvh = (int)(t % sides) % p.a.Hkv;
        int first, last, row0, pi, npages;   // slots [first, last) get rows row0, row0 + 1, ...
        const int32_t* pages;
        if (b < p.block0[p.a.nchunks]) {
            int P = p.a.cP[0], C = p.cC[0], r = 0, at = 0, page0 = 0, page1 = p.a.cPage0[1];
#pragma unroll
            for (int j = 1; j < kMaxChunks; ++j)
                if (j < p.a.nchunks && b >= p.block0[j]) {
                    P = p.a.cP[j], C = p.cC[j], r = p.a.cRow0[j], at = p.block0[j], page0 = p.a.cPage0[j], page1 = p.a.cPage0[j + 1];
                }
            pi = P / kPageSize + b - at;
            first = max(P - pi * kPageSize, 0);
            last = min(P + C - pi * kPageSize, kPageSize);
            row0 = r + pi * kPageSize + first - P;
            pages = p.a.prefill_pages + page0;
            npages = page1 - page0;
        } else {
            const int i = b - p.block0[p.a.nchunks], len = p.a.decode_kv_len[i], beg = p.a.decode_page_indptr[i];
            npages = p.a.decode_page_indptr[i + 1] - beg;
            pages = p.a.decode_pages + beg;
            pi = len < 1 ? npages : (len - 1) / kPageSize;
            first = (len - 1) % kPageSize;
            last = first + 1;
            row0 = p.a.C + i;
        }
        if (pi >= npages) {
            if (lane == 0) report(p.a.ctrl, SW_ERR_OUT_OF_RANGE, kSiteAppendLen, row0);
            continue;
        }
        const int page = pages[pi];
        const __nv_bfloat16* src = (side ? p.a.v_new : p.a.k_new) + ((int64_t)row0 * p.a.Hkv + kvh) * D + col;
        uint4 x[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * kRows + sub;
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            if (slot >= first && slot < last) x[i] = *reinterpret_cast<const uint4*>(src + (int64_t)(slot - first) * p.a.Hkv * D);
        }
        if (page < 0 || (int64_t)page >= p.a.num_pages) {
            if (lane == 0) report(p.a.ctrl, SW_ERR_OUT_OF_RANGE, kSiteAppendPage, row0);
            continue;
        }
        const int64_t block = ((int64_t)page * 2 + side) * p.a.Hkv + kvh;
        const float before = first > 0 ? p.scales[block] : 0.f;
        uint32_t top2 = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
        const uint32_t top = __reduce_max_sync(0xffffffffu, max(top2 & 0xffffu, top2 >> 16));
        // 448 = 1.75 * 2^8: the exponent of the largest value less 8, and one more where its mantissa is above 0.75
        const int e = max((int)(top >> 7) - 127 - 8 + ((top & 127) > 96), kMinScaleExp);
        float scale = top >= 0x7f80u ? __int_as_float(0x7fc00000) : __int_as_float((e + 127) << 23);
        if (!(scale <= before)) {   // (also where the new scale is NaN)
            if (first > 0 && !(before != before)) {   // the rows in front of the new ones move to the larger scale
                const float f = before / scale;
                uint8_t* dst = p.pool + block * kPageSize * D;
                for (int c = lane; c < first * (D / 16); c += 32) {
                    uint4 w = *reinterpret_cast<const uint4*>(dst + c * 16);
                    w = make_uint4(rescale_e4m3x4(w.x, f), rescale_e4m3x4(w.y, f), rescale_e4m3x4(w.z, f), rescale_e4m3x4(w.w, f));
                    *reinterpret_cast<uint4*>(dst + c * 16) = w;
                }
            } else if (first > 0) {
                scale = before;   // NaN stays
            }
            if (lane == 0) p.scales[block] = scale;
        } else {
            scale = before;
        }
        const float f = 1.f / scale;   // a power of two
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * kRows + sub;
            if (slot >= first && slot < last)
                *reinterpret_cast<uint2*>(p.pool + (block * kPageSize + slot) * D + col) =
                    make_uint2(e4m3x4_of(bf16_lo(x[i].x) * f, bf16_hi(x[i].x) * f, bf16_lo(x[i].y) * f, bf16_hi(x[i].y) * f),
                               e4m3x4_of(bf16_lo(x[i].z) * f, bf16_hi(x[i].z) * f, bf16_lo(x[i].w) * f, bf16_hi(x[i].w) * f));
        }
    }
}

// The prompts of the iteration's chunks as bf16 pages 0, 1, ... of `copy`, one prompt behind the other, and the list of those pages: what the
// chunk-prefill tiles read in place of the 8-bit pool where that is faster (chunks_copied).  One warp per block, 8 bytes a lane and load;
// slots at or past the prompt's end become zeros.  Exact: e4m3 times a power of two is a bf16 number.  An e4m3 is a bf16 whose exponent is 120
// too small once its seven lower bits are moved up by four, subnormal values included; one product with 2^120 times the scale does the rest.
template <int D>
__global__ void __launch_bounds__(kKv8Threads) sw_kv8_expand_kernel(const Kv8Params p) {
    constexpr int kLoads = D / 16, kRowLanes = D / 8;
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, sides = 2 * p.a.Hkv;
    const int64_t tasks = (int64_t)p.block0[p.a.nchunks] * sides;
    for (int64_t t = (int64_t)blockIdx.x * (kKv8Threads / 32) + threadIdx.x / 32; t < tasks; t += (int64_t)gridDim.x * (kKv8Threads / 32)) {
        const int b = (int)(t / sides), hs = (int)(t % sides);
        int end = p.a.cP[0] + p.cC[0], at = 0, page0 = 0;
#pragma unroll
        for (int j = 1; j < kMaxChunks; ++j)
            if (j < p.a.nchunks && b >= p.block0[j]) end = p.a.cP[j] + p.cC[j], at = p.block0[j], page0 = p.a.cPage0[j];
        int page = p.a.prefill_pages[page0 + b - at];
        if (page < 0 || (int64_t)page >= p.a.num_pages) {
            if (lane == 0) report(p.a.ctrl, SW_ERR_OUT_OF_RANGE, kSiteAttnPage, b);
            page = 0;
        }
        const int valid = end - (b - at) * kPageSize;
        const int64_t block = (int64_t)page * sides + hs;
        const uint2* src = reinterpret_cast<const uint2*>(p.pool + block * kPageSize * D) + lane;
        uint4* dst = reinterpret_cast<uint4*>(p.copy + ((int64_t)b * sides + hs) * kPageSize * D) + lane;
        uint2 w[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) w[i] = __ldcs(src + i * 32);
        const float scale = p.scales[block], rest = scale > 128.f ? scale * 0.0078125f : 1.f;   // 2^127 is as far as one factor goes
        const float f = (scale > 128.f ? 128.f : scale) * 1.329227995784916e36f;   // 2^120
        const uint32_t factor = pack_bf16x2(f, f), more = pack_bf16x2(rest, rest);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {   // bytes 2 e and 2 e + 1, each with eight copies of its sign above it
                asm("prmt.b32 %0, %1, %1, %2;" : "=r"(x[e]) : "r"(e < 2 ? w[i].x : w[i].y), "r"(e & 1 ? 0xb3a2 : 0x9180));
                x[e] = (x[e] << 4) & 0x87f087f0u;
                asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(x[e]) : "r"(x[e]), "r"(factor));
                if (rest != 1.f) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(x[e]) : "r"(x[e]), "r"(more));
            }
            // the codes 0x7f and 0xff, which this made 480 times the scale, stand for NaN
            if ((((w[i].x & 0x7f7f7f7fu) + 0x01010101u) | ((w[i].y & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t two = (e < 2 ? w[i].x : w[i].y) >> 16 * (e & 1);
                    if ((two & 0x7fu) == 0x7fu) x[e] |= 0x7fffu;
                    if ((two & 0x7f00u) == 0x7f00u) x[e] |= 0x7fff0000u;
                }
            }
            dst[i * 32] = (i * 32 + lane) / kRowLanes < valid ? make_uint4(x[0], x[1], x[2], x[3]) : make_uint4(0u, 0u, 0u, 0u);
        }
        if (hs == 0 && lane == 0) p.list[b] = b;
    }
}

namespace {
template <class K>
cudaError_t launch_blocks(K* kernel, const Kv8Params& p, int64_t tasks, int num_sms, cudaStream_t stream) {
    const int64_t blocks = (tasks + kKv8Threads / 32 - 1) / (kKv8Threads / 32);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks < (int64_t)num_sms * 4 ? blocks : (int64_t)num_sms * 4));   // resident at once
    cfg.blockDim = dim3(kKv8Threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}
}  // namespace

cudaError_t launch_kv8_append(const AppendParams& a, const int* cC, uint8_t* pool, float* scales, int num_sms, cudaStream_t stream) {
    Kv8Params p{};
    p.a = a;
    p.pool = pool;
    p.scales = scales;
    for (int j = 0; j < a.nchunks; ++j) {
        p.cC[j] = cC[j];
        p.block0[j + 1] = p.block0[j] + (int)(((int64_t)a.cP[j] + cC[j] - 1) / kPageSize) - a.cP[j] / kPageSize + 1;
    }
    const int64_t tasks = (int64_t)(p.block0[a.nchunks] + a.n) * 2 * a.Hkv;
    return a.D == 64 ? launch_blocks(sw_kv8_append_kernel<64>, p, tasks, num_sms, stream)
                     : launch_blocks(sw_kv8_append_kernel<128>, p, tasks, num_sms, stream);
}

cudaError_t launch_kv8_expand(const AppendParams& a, const int* cC, const uint8_t* pool, const float* scales, __nv_bfloat16* copy, int32_t* list,
                              int num_sms, cudaStream_t stream) {
    Kv8Params p{};
    p.a = a;
    p.pool = const_cast<uint8_t*>(pool);
    p.scales = const_cast<float*>(scales);
    p.copy = copy;
    p.list = list;
    for (int j = 0; j < a.nchunks; ++j) {
        p.cC[j] = cC[j];
        p.block0[j + 1] = p.block0[j] + (int)(((int64_t)a.cP[j] + cC[j] - 1) / kPageSize) + 1;
    }
    const int64_t tasks = (int64_t)p.block0[a.nchunks] * 2 * a.Hkv;
    return a.D == 64 ? launch_blocks(sw_kv8_expand_kernel<64>, p, tasks, num_sms, stream)
                     : launch_blocks(sw_kv8_expand_kernel<128>, p, tasks, num_sms, stream);
}

cudaError_t configure_kv8_kernels(int head_dim) { return configure_option<kKv8>(head_dim); }
cudaError_t launch_kv8_attn(int head_dim, bool copied, const KvMaps& kv_maps, const CUtensorMap& q_map, const CUtensorMap& out_map,
                            const MixedParams& p, int num_sms, cudaStream_t stream) {
    return copied ? launch_option<kKv8, kPlain>(head_dim, kv_maps, q_map, out_map, p, num_sms, stream)
                  : launch_option<kKv8>(head_dim, kv_maps, q_map, out_map, p, num_sms, stream);
}

}  // namespace sw
