// C-ABI entry points of the device path: context, KV append, the mixed attention launch, the host-buffer
// iteration and the cost probe.  Host code only validates, marshals and launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

#include "sw.h"
#include "sw_error.h"
#include "sw_internal.h"

namespace {

using sw::EncodeTiledFn;

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Offsets of the regions inside the caller's workspace.
struct WsLayout {
    size_t ctrl, tickets, part_ml, part_o, pf_tickets, pf_ml, pf_o, st_q, st_k, st_v, st_out, st_lse, st_pages, total;
    int pf_slots;
    int max_items;
};

bool layout_supported(const sw_layout& l) {
    if (l.num_q_heads <= 0 || l.num_kv_heads <= 0 || l.num_pages <= 0) return false;
    if (l.head_dim != 64 && l.head_dim != 128) return false;
    if (l.page_size != sw::kPageSize) return false;
    if (l.num_q_heads % l.num_kv_heads != 0) return false;
    const int g = l.num_q_heads / l.num_kv_heads;
    if (!(g == 1 || g == 2 || g == 4 || g == 8)) return false;
    if (l.num_pages > (int64_t)1 << 30) return false;
    if (2 * l.num_pages * l.num_kv_heads >= (int64_t)1 << 31) return false;  // (page, K|V, head) blocks are int32 coordinates
    return true;
}

WsLayout ws_layout(const sw_layout& l, int max_chunk, int max_decode, int64_t max_pages) {
    WsLayout w{};
    const int g = l.num_q_heads / l.num_kv_heads;
    const size_t rows = (size_t)max_chunk + max_decode;
    w.max_items = sw::kTargetItems + max_decode * l.num_kv_heads;
    size_t off = 0;
    w.ctrl = off;     off = align_up(off + sw::kCtrWords * 4, 256);
    w.tickets = off;  off = align_up(off + (size_t)std::max(1, max_decode) * l.num_kv_heads * 4 * 2, 256);  // tickets, ready
    w.part_ml = off;  off = align_up(off + (size_t)w.max_items * 2 * sw::kMaxGroup * 4, 256);
    w.part_o = off;   off = align_up(off + (size_t)w.max_items * g * l.head_dim * 4, 256);
    // 256-row groups of the chunks of one iteration: every chunk may end in a ragged group
    const size_t groups = ((size_t)max_chunk + (256 / g) - 1) / (256 / g) + sw::kMaxChunks;
    w.pf_tickets = off; off = align_up(off + std::max<size_t>(1, groups) * l.num_kv_heads * 2 * 4, 256);
    // pieces of items publish partial results: one slot per CTA, more where a single chunk can hold a whole round of
    // items (its leftover items may then be cut into pieces that run in several rounds; the plan never uses more slots
    // than it is given)
    const size_t single_chunk_items = ((size_t)max_chunk + (256 / g) - 1) / (256 / g) * l.num_kv_heads;
    w.pf_slots = single_chunk_items >= 96 ? sw::kPfRoundSlots : sw::kMaxCtas;
    w.pf_ml = off;    off = align_up(off + (size_t)w.pf_slots * 2 * 256 * 4, 256);
    w.pf_o = off;     off = align_up(off + (max_chunk > 0 ? (size_t)w.pf_slots * 2 * 128 * l.head_dim * 4 : 0), 256);
    w.st_q = off;     off = align_up(off + rows * l.num_q_heads * l.head_dim * 2, 256);
    w.st_k = off;     off = align_up(off + rows * l.num_kv_heads * l.head_dim * 2, 256);
    w.st_v = off;     off = align_up(off + rows * l.num_kv_heads * l.head_dim * 2, 256);
    w.st_out = off;   off = align_up(off + rows * l.num_q_heads * l.head_dim * 2, 256);
    w.st_lse = off;   off = align_up(off + rows * l.num_q_heads * 4, 256);
    w.st_pages = off; off = align_up(off + ((size_t)max_pages + 2 * (size_t)max_decode + 8) * 4, 256);
    w.total = off;
    return w;
}

}  // namespace

// Host-buffer iterations of kHostPartBytes of inputs or more are run in parts, so that one part's launch runs beside the next one's
// copies.  Two parts: more of them cost more calls and launches than they hide (576 rows of 12 KB: 320 us whole, 297 in two parts,
// 312 in three or four).
constexpr int kHostParts = 2;
constexpr size_t kHostPartBytes = 4u << 20;

struct sw_ctx {
    sw_layout layout;
    bool window_grid_resident = false;   // as grid_resident, of the kernels with a window
    int device = 0;
    int num_sms = 0;
    float stage_us = 0.f, step_us = 0.f;  // planning estimates from the device's clocks (sw::device_timing)
    long long line_wait_cycles = sw::kLineWaitCycles;
    bool grid_resident = false;  // the persistent grid fits the device at once (needed by the fused append + attention launch)
    int max_chunk = 0, max_decode = 0;
    int64_t max_pages = 0;
    uint8_t* ws = nullptr;
    WsLayout w{};
    EncodeTiledFn encode = nullptr;
    struct MapEntry {
        const void* pool;
        sw::KvMaps maps;
    };
    std::vector<MapEntry> kv_maps;  // small cache: one entry per pool of a layer stack
    struct Kv8MapEntry {
        const void* pool;
        sw::KvMaps maps;
    };
    Kv8MapEntry kv8_maps[128];   // likewise of 8-bit pools, the oldest replaced first
    int kv8_map_count = 0, kv8_map_next = 0;
    cudaEvent_t ev0 = nullptr, ev1 = nullptr;
    // host-buffer iterations in parts: the copies' stream and events
    cudaStream_t copies = nullptr;
    cudaEvent_t ev_start = nullptr, ev_up = nullptr, ev_done[kHostParts + 1] = {};   // the last one: the decode rows
};

namespace {

#define SW_CUDA(call)                                                                                        \
    do {                                                                                                     \
        cudaError_t e_ = (call);                                                                             \
        if (e_ != cudaSuccess) return sw_fail(SW_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e_));  \
    } while (0)

// Launching calls run on the caller's current device: a context serves the device it was created on and refuses any other
// (its workspace, tensor maps and kernel attributes belong to that device).
sw_status check_current_device(const sw_ctx* ctx, const char* who) {
    int current = -1;
    SW_CUDA(cudaGetDevice(&current));
    if (current != ctx->device)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: the context belongs to device %d but device %d is current", who, ctx->device,
                       current);
    return SW_OK;
}

sw_status kv_map_for(sw_ctx* ctx, const void* pool, const sw::KvMaps** out) {
    for (auto& e : ctx->kv_maps)
        if (e.pool == pool) {
            *out = &e.maps;
            return SW_OK;
        }
    const sw_layout& l = ctx->layout;
    if ((reinterpret_cast<uintptr_t>(pool) & 15) != 0) return sw_fail(SW_ERR_INVALID_ARG, "kv_pool must be 16-byte aligned");
    sw_ctx::MapEntry e;
    e.pool = pool;
    CUresult r = sw::encode_kv_maps(ctx->encode, l, pool, &e.maps);
    if (r != CUDA_SUCCESS) return sw_fail(SW_ERR_CUDA, "cuTensorMapEncodeTiled(kv pool) failed with CUresult %d", (int)r);
    if (ctx->kv_maps.size() >= 128) ctx->kv_maps.erase(ctx->kv_maps.begin());
    ctx->kv_maps.push_back(e);
    *out = &ctx->kv_maps.back().maps;
    return SW_OK;
}

// The prefill chunks of a batch in the form the kernels take (single-chunk batches become one chunk).
struct Chunks {
    int n = 0;
    int rows = 0;  // chunk rows of the iteration = sum of the chunk lengths
    int P[sw::kMaxChunks] = {}, C[sw::kMaxChunks] = {}, row0[sw::kMaxChunks] = {}, page0[sw::kMaxChunks + 1] = {};
};
static_assert(SW_MAX_CHUNKS == sw::kMaxChunks, "the header states the limit");

sw_status chunks_of(const sw_batch* b, const char* who, Chunks* out) {
    Chunks c;
    if (b->num_chunks < 0 || b->num_chunks > sw::kMaxChunks)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: num_chunks %d outside 0..%d", who, b->num_chunks, sw::kMaxChunks);
    if (b->num_chunks == 0) {
        if (b->chunk_len > 0) {
            c.n = 1;
            c.P[0] = b->prefix_len;
            c.C[0] = b->chunk_len;
            c.rows = b->chunk_len;
            c.page0[1] = b->num_prefill_pages;
        }
    } else {
        if (!b->chunk_prefix_lens || !b->chunk_lens || !b->chunk_page_indptr)
            return sw_fail(SW_ERR_INVALID_ARG, "%s: chunk arrays missing", who);
        int64_t rows = 0;
        for (int j = 0; j < b->num_chunks; ++j) {
            if (b->chunk_prefix_lens[j] < 0 || b->chunk_lens[j] < 1)
                return sw_fail(SW_ERR_INVALID_ARG, "%s: chunk %d has prefix %d and length %d", who, j, b->chunk_prefix_lens[j],
                               b->chunk_lens[j]);
            if (b->chunk_page_indptr[j + 1] < b->chunk_page_indptr[j] || b->chunk_page_indptr[0] != 0)
                return sw_fail(SW_ERR_INVALID_ARG, "%s: chunk_page_indptr must start at 0 and not decrease", who);
            c.P[j] = b->chunk_prefix_lens[j];
            c.C[j] = b->chunk_lens[j];
            c.row0[j] = (int)rows;
            c.page0[j] = b->chunk_page_indptr[j];
            rows += b->chunk_lens[j];
            if (rows > sw::kMaxChunk) return sw_fail(SW_ERR_UNSUPPORTED, "%s: more than %d chunk rows", who, sw::kMaxChunk);
        }
        c.n = b->num_chunks;
        c.rows = (int)rows;
        c.page0[c.n] = b->chunk_page_indptr[c.n];
        if (c.page0[c.n] != b->num_prefill_pages)
            return sw_fail(SW_ERR_INVALID_ARG, "%s: chunk_page_indptr ends at %d, num_prefill_pages is %d", who, c.page0[c.n],
                           b->num_prefill_pages);
    }
    for (int j = c.n; j <= sw::kMaxChunks; ++j) c.page0[j] = c.page0[c.n];
    *out = c;
    return SW_OK;
}

// cross: a chunk's keys are its prefix alone, and there may be none, nor pages.
sw_status check_batch(const sw_ctx* ctx, const sw_batch* b, const char* who, Chunks* chunks, bool cross = false) {
    if (!ctx || !b) return sw_fail(SW_ERR_INVALID_ARG, "%s: null context or batch", who);
    if (b->prefix_len < 0 || b->chunk_len < 0 || b->num_decode < 0 || b->num_prefill_pages < 0)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: negative size in batch", who);
    sw_status cs = chunks_of(b, who, chunks);
    if (cs != SW_OK) return cs;
    if (chunks->rows > ctx->max_chunk || b->num_decode > ctx->max_decode)
        return sw_fail(SW_ERR_WORKSPACE, "%s: %d chunk rows / num_decode %d exceed the context's limits %d / %d", who,
                       chunks->rows, b->num_decode, ctx->max_chunk, ctx->max_decode);
    if (b->num_decode > sw::kMaxDecode)
        return sw_fail(SW_ERR_UNSUPPORTED, "%s: at most %d decode requests per iteration", who, sw::kMaxDecode);
    for (int j = 0; j < chunks->n; ++j) {
        const int64_t need = ((int64_t)chunks->P[j] + (cross ? 0 : chunks->C[j]) + sw::kPageSize - 1) / sw::kPageSize;
        const int have = chunks->page0[j + 1] - chunks->page0[j];
        if ((!b->prefill_pages && need > 0) || have < need)
            return sw_fail(SW_ERR_OUT_OF_RANGE, "%s: prefill page list has %d entries, %s needs %lld", who, have, cross ? "P" : "P+C",
                           (long long)need);
    }
    if (b->num_decode > 0 && (!b->decode_kv_len || !b->decode_page_indptr || (!b->decode_pages && !cross)))
        return sw_fail(SW_ERR_INVALID_ARG, "%s: decode arrays missing", who);
    return SW_OK;
}

}  // namespace

namespace {
// What a context asks of its device.  The driver takes 1.2 ms for each clock rate (and 2.5 for all properties at once, which are not asked for), so a process asks
// once per device: a context is created in 20 to 35 us (80 where it gets the streams of host-buffer iterations) instead of 5 ms.
struct DeviceFacts {
    int major, minor, sms, mem_khz, bus_bits, sm_khz;
};
sw_status device_facts(int device, DeviceFacts* out) {
    constexpr int kMost = 64;
    static DeviceFacts kept[kMost];
    static std::atomic<int> state[kMost];   // 0: nothing; 1: being written; 2: there
    const bool keeps = device >= 0 && device < kMost;
    if (keeps && state[device].load(std::memory_order_acquire) == 2) {
        *out = kept[device];
        return SW_OK;
    }
    DeviceFacts f{};
    const struct {
        cudaDeviceAttr attr;
        int* to;
    } asked[] = {{cudaDevAttrComputeCapabilityMajor, &f.major}, {cudaDevAttrComputeCapabilityMinor, &f.minor}, {cudaDevAttrMultiProcessorCount, &f.sms},
                 {cudaDevAttrMemoryClockRate, &f.mem_khz}, {cudaDevAttrGlobalMemoryBusWidth, &f.bus_bits}, {cudaDevAttrClockRate, &f.sm_khz}};
    for (const auto& a : asked) SW_CUDA(cudaDeviceGetAttribute(a.to, a.attr, device));
    int nothing = 0;
    if (keeps && state[device].compare_exchange_strong(nothing, 1, std::memory_order_relaxed)) {   // (of several threads one keeps what all have found)
        kept[device] = f;
        state[device].store(2, std::memory_order_release);
    }
    *out = f;
    return SW_OK;
}

sw_status make_copy_stream(sw_ctx* ctx) {
    SW_CUDA(cudaStreamCreateWithFlags(&ctx->copies, cudaStreamNonBlocking));
    SW_CUDA(cudaEventCreateWithFlags(&ctx->ev_start, cudaEventDisableTiming));
    SW_CUDA(cudaEventCreateWithFlags(&ctx->ev_up, cudaEventDisableTiming));
    for (cudaEvent_t& e : ctx->ev_done)
        SW_CUDA(cudaEventCreateWithFlags(&e, cudaEventDisableTiming));
    return SW_OK;
}
}  // namespace

extern "C" {

size_t sw_workspace_bytes(const sw_layout* layout, int32_t max_chunk, int32_t max_decode, int64_t max_pages) {
    if (!layout || !layout_supported(*layout) || max_chunk < 0 || max_decode < 0 || max_pages < 0 ||
        max_decode > sw::kMaxDecode || max_chunk > sw::kMaxChunk)
        return 0;
    return ws_layout(*layout, max_chunk, max_decode, max_pages).total;
}

sw_status sw_create(const sw_layout* layout, int device, void* workspace, size_t workspace_bytes, int32_t max_chunk,
                    int32_t max_decode, int64_t max_pages, sw_ctx** out) {
    if (!layout || !out) return sw_fail(SW_ERR_INVALID_ARG, "sw_create: null argument");
    if (!layout_supported(*layout))
        return sw_fail(SW_ERR_UNSUPPORTED,
                       "sw_create: supported shapes are head_dim 64|128, page_size 16, q/kv head ratio 1|2|4|8");
    if (max_chunk < 0 || max_decode < 0 || max_pages < 0 || max_decode > sw::kMaxDecode || max_chunk > sw::kMaxChunk)
        return sw_fail(SW_ERR_INVALID_ARG, "sw_create: limits out of range (max_decode <= %d, max_chunk <= %d)", sw::kMaxDecode,
                       sw::kMaxChunk);
    const WsLayout w = ws_layout(*layout, max_chunk, max_decode, max_pages);
    if (!workspace || workspace_bytes < w.total || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
        return sw_fail(SW_ERR_WORKSPACE, "sw_create: workspace must be 256-byte aligned and hold %zu bytes", w.total);
    DeviceFacts facts;
    const sw_status known = device_facts(device, &facts);
    if (known != SW_OK) return known;
    if (facts.major != 10)
        return sw_fail(SW_ERR_UNSUPPORTED, "sw_create: device %d is compute capability %d.%d; this library is sm_100a only",
                       device, facts.major, facts.minor);
    // the set-up below runs with `device` current; the caller's current device is put back before returning
    int caller_device = device;
    SW_CUDA(cudaGetDevice(&caller_device));
    struct Restore {
        int dev, want;
        ~Restore() {
            if (dev != want) cudaSetDevice(dev);
        }
    } restore{caller_device, device};
    if (caller_device != device) SW_CUDA(cudaSetDevice(device));
    sw_ctx* ctx = new (std::nothrow) sw_ctx();
    if (!ctx) return sw_fail(SW_ERR_INVALID_ARG, "sw_create: out of host memory");
    ctx->layout = *layout;
    if (ctx->layout.sm_scale <= 0.f) ctx->layout.sm_scale = 1.0f / std::sqrt((float)layout->head_dim);
    ctx->device = device;
    ctx->num_sms = std::min(facts.sms, sw::kMaxCtas);
    sw::device_timing(facts.mem_khz, facts.bus_bits, facts.sm_khz, layout->head_dim, &ctx->stage_us, &ctx->step_us);
    ctx->max_chunk = max_chunk;
    ctx->max_decode = max_decode;
    ctx->max_pages = max_pages;
    ctx->ws = static_cast<uint8_t*>(workspace);
    ctx->w = w;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn) {
        delete ctx;
        return sw_fail(SW_ERR_CUDA, "sw_create: cuTensorMapEncodeTiled is not available from the driver");
    }
    ctx->encode = reinterpret_cast<EncodeTiledFn>(fn);
    e = cudaMemset(ctx->ws, 0, w.pf_ml);  // control words, tickets and split-KV scratch start at zero
    if (e == cudaSuccess) e = sw::configure_kernels(layout->head_dim);
    if (e == cudaSuccess) e = sw::configure_window_kernels(layout->head_dim);
    if (e == cudaSuccess) e = sw::configure_kv8_kernels(layout->head_dim);
    if (e == cudaSuccess) e = sw::configure_scored_kernels(layout->head_dim);
    if (e == cudaSuccess) e = sw::configure_evict_kernels();
    if (e == cudaSuccess) e = sw::configure_cross_kernels(layout->head_dim);
    if (e == cudaSuccess) e = sw::configure_sample_kernels();
    int per_sm = 0, window_per_sm = 0;
    if (e == cudaSuccess) e = sw::mixed_attn_resident_ctas_per_sm(layout->head_dim, &per_sm);
    if (e == cudaSuccess) e = sw::window_attn_resident_ctas_per_sm(layout->head_dim, &window_per_sm);
    ctx->window_grid_resident = (int64_t)window_per_sm * facts.sms >= ctx->num_sms;
    // The fused launch lets CTAs wait for one another's share of the KV append, so the whole grid has to be resident.
    // Where it would not be (fewer SMs than the properties promise cannot be seen here, but a smaller shared-memory
    // or register budget can) sw_mixed_iteration_run issues the append as a launch of its own.
    ctx->grid_resident = (int64_t)per_sm * facts.sms >= ctx->num_sms;
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        delete ctx;
        return sw_fail(SW_ERR_CUDA, "sw_create: device set-up failed: %s", cudaGetErrorString(e));
    }
    if (max_pages > 0) {   // the context may take host-buffer iterations (0.1 ms here rather than in the first of them)
        const sw_status st = make_copy_stream(ctx);
        if (st != SW_OK) {
            sw_destroy(ctx);
            return st;
        }
    }
    *out = ctx;
    return SW_OK;
}

void sw_destroy(sw_ctx* ctx) {
    if (!ctx) return;
    if (ctx->ev0) cudaEventDestroy(ctx->ev0);
    if (ctx->ev1) cudaEventDestroy(ctx->ev1);
    if (ctx->copies) cudaStreamDestroy(ctx->copies);
    if (ctx->ev_start) cudaEventDestroy(ctx->ev_start);
    if (ctx->ev_up) cudaEventDestroy(ctx->ev_up);
    for (cudaEvent_t e : ctx->ev_done)
        if (e) cudaEventDestroy(e);
    delete ctx;
}

namespace {
sw::AppendParams append_params(const sw_ctx* ctx, const sw_batch* batch, const Chunks& ch, void* kv_pool, const void* k_new, const void* v_new) {
    sw::AppendParams p{};
    p.Hkv = ctx->layout.num_kv_heads;
    p.D = ctx->layout.head_dim;
    p.num_pages = ctx->layout.num_pages;
    p.C = ch.rows;
    p.n = batch->num_decode;
    p.nchunks = ch.n;
    std::memcpy(p.cP, ch.P, sizeof p.cP);
    std::memcpy(p.cRow0, ch.row0, sizeof p.cRow0);
    std::memcpy(p.cPage0, ch.page0, sizeof p.cPage0);
    p.prefill_pages = batch->prefill_pages;
    p.num_prefill_pages = batch->num_prefill_pages;
    p.decode_kv_len = batch->decode_kv_len;
    p.decode_page_indptr = batch->decode_page_indptr;
    p.decode_pages = batch->decode_pages;
    p.k_new = static_cast<const __nv_bfloat16*>(k_new);
    p.v_new = static_cast<const __nv_bfloat16*>(v_new);
    p.pool = static_cast<__nv_bfloat16*>(kv_pool);
    p.ctrl = reinterpret_cast<int32_t*>(ctx->ws + ctx->w.ctrl);
    return p;
}
}  // namespace

sw_status sw_kv_append(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, const void* k_new, const void* v_new,
                       void* stream) {
    Chunks ch;
    sw_status st = check_batch(ctx, batch, "sw_kv_append", &ch);
    if (st != SW_OK) return st;
    if (ch.rows + batch->num_decode == 0) return SW_OK;
    if (!kv_pool || !k_new || !v_new) return sw_fail(SW_ERR_INVALID_ARG, "sw_kv_append: null tensor");
    st = check_current_device(ctx, "sw_kv_append");
    if (st != SW_OK) return st;
    if (((reinterpret_cast<uintptr_t>(kv_pool) | reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new)) & 15) != 0)
        return sw_fail(SW_ERR_INVALID_ARG, "sw_kv_append: tensors must be 16-byte aligned");
    const sw::AppendParams p = append_params(ctx, batch, ch, kv_pool, k_new, v_new);
    SW_CUDA(sw::launch_kv_append(p, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

namespace {
// The parameters of an attention launch that do not depend on what the pool holds.
sw::MixedParams mixed_params(const sw_ctx* ctx, const sw_batch* batch, const Chunks& ch, const void* q, void* out, float* lse) {
    const sw_layout& l = ctx->layout;
    sw::MixedParams p{};
    p.Hq = l.num_q_heads;
    p.Hkv = l.num_kv_heads;
    p.group = l.num_q_heads / l.num_kv_heads;
    p.num_pages = p.chunk_pool_pages = l.num_pages;
    p.sm_scale = l.sm_scale;
    p.sm_scale_log2 = l.sm_scale * 1.4426950408889634f;
    p.stage_us = ctx->stage_us;
    p.step_us = ctx->step_us;
    p.stages_per_us = 1.f / ctx->stage_us;
    p.steps_per_stage = ctx->stage_us / ctx->step_us;
    sw::small_batch_limits(batch->num_decode, l.num_kv_heads, ctx->num_sms, &p.small_from, &p.small_to);
    p.C = ch.rows;
    p.n = batch->num_decode;
    p.nchunks = ch.n;
    std::memcpy(p.cP, ch.P, sizeof p.cP);
    std::memcpy(p.cC, ch.C, sizeof p.cC);
    std::memcpy(p.cRow0, ch.row0, sizeof p.cRow0);
    std::memcpy(p.cPage0, ch.page0, sizeof p.cPage0);
    p.prefill_pages = batch->prefill_pages;
    p.num_prefill_pages = batch->num_prefill_pages;
    p.decode_kv_len = batch->decode_kv_len;
    p.decode_page_indptr = batch->decode_page_indptr;
    p.decode_pages = batch->decode_pages;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.out = static_cast<__nv_bfloat16*>(out);
    p.lse = lse;
    p.ctrl = reinterpret_cast<int32_t*>(ctx->ws + ctx->w.ctrl);
    p.tickets = reinterpret_cast<int32_t*>(ctx->ws + ctx->w.tickets);
    p.ready = p.tickets + (size_t)std::max(1, ctx->max_decode) * l.num_kv_heads;
    p.part_ml = reinterpret_cast<float*>(ctx->ws + ctx->w.part_ml);
    p.part_o = reinterpret_cast<float*>(ctx->ws + ctx->w.part_o);
    p.max_items = ctx->w.max_items;
    p.target_items = sw::kTargetItems;
    p.line_wait_cycles = ctx->line_wait_cycles;
    p.pf_ml = reinterpret_cast<float*>(ctx->ws + ctx->w.pf_ml);
    p.pf_o = reinterpret_cast<float*>(ctx->ws + ctx->w.pf_o);
    p.pf_slots = ctx->w.pf_slots;
    p.pf_tickets = reinterpret_cast<int32_t*>(ctx->ws + ctx->w.pf_tickets);
    return p;
}

// q as [row][head][element] restricted to the chunk rows: one box = 128 tile rows (token-major, the g heads of a
// KV head minor) x 64 elements; rows past the chunk read as zero.  out has the same shape: tiles whose 128 rows all lie inside a chunk
// are stored through its map.  (Without chunk rows the maps are left as they are.)
sw_status encode_row_maps(const sw_ctx* ctx, const sw::MixedParams& p, CUtensorMap* q_map, CUtensorMap* out_map) {
    if (p.C == 0) return SW_OK;
    const sw_layout& l = ctx->layout;
    const cuuint64_t dims[3] = {(cuuint64_t)l.head_dim, (cuuint64_t)l.num_q_heads, (cuuint64_t)p.C};
    const cuuint64_t strides[2] = {(cuuint64_t)l.head_dim * 2, (cuuint64_t)l.num_q_heads * l.head_dim * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)p.group, (cuuint32_t)(128 / p.group)};
    const cuuint32_t elem_strides[3] = {1, 1, 1};
    CUresult r = ctx->encode(q_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(p.q), dims, strides, box,
                             elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return sw_fail(SW_ERR_CUDA, "cuTensorMapEncodeTiled(q) failed with CUresult %d", (int)r);
    r = ctx->encode(out_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.out, dims, strides, box, elem_strides,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return sw_fail(SW_ERR_CUDA, "cuTensorMapEncodeTiled(out) failed with CUresult %d", (int)r);
    return SW_OK;
}

bool aligned16(const void* a, const void* b = nullptr, const void* c = nullptr, const void* d = nullptr) {
    return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c) | reinterpret_cast<uintptr_t>(d)) & 15) == 0;
}

// The last `keys` keys and the first `sinks` are attended; keys == 0: all.
struct Window {
    int keys = 0, sinks = 0;
};
sw_status check_window(int32_t window, int32_t sinks, const char* who, Window* out) {
    if (window < 1 || sinks < 0) return sw_fail(SW_ERR_INVALID_ARG, "%s: window %d, sinks %d (at least 1 and 0)", who, window, sinks);
    out->keys = std::min(window, 1 << 30);   // (longer than any context whose positions the kernels can add to it)
    out->sinks = std::min(sinks, 1 << 30);
    return SW_OK;
}

// The attention launch; with k_new / v_new non-null the same launch first writes those rows into the pool.
sw_status run_mixed(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, const void* k_new, const void* v_new, const void* q,
                    void* out, float* lse, void* stream, const char* who, Window window = {}) {
    Chunks ch;
    sw_status st = check_batch(ctx, batch, who, &ch);
    if (st != SW_OK) return st;
    if (ch.rows + batch->num_decode == 0) return SW_OK;
    if (!kv_pool || !q || !out) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    if (!aligned16(q, out, k_new, v_new)) return sw_fail(SW_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned", who);
    const sw::KvMaps* kv_maps = nullptr;
    st = kv_map_for(ctx, kv_pool, &kv_maps);
    if (st != SW_OK) return st;
    sw::MixedParams p = mixed_params(ctx, batch, ch, q, out, lse);
    if (k_new) {
        p.k_new = static_cast<const __nv_bfloat16*>(k_new);
        p.v_new = static_cast<const __nv_bfloat16*>(v_new);
        p.pool = static_cast<__nv_bfloat16*>(kv_pool);
        p.append_first = p.C > 0;
        p.append_last = p.C == 0;
    }
    CUtensorMap q_map = kv_maps->half, out_map = kv_maps->half;
    st = encode_row_maps(ctx, p, &q_map, &out_map);
    if (st != SW_OK) return st;
    if (window.keys > 0) {
        p.window = window.keys;
        p.sinks = window.sinks;
        p.sink_pages = (window.sinks + sw::kPageSize - 1) / sw::kPageSize;
        SW_CUDA(sw::launch_window_attn(ctx->layout.head_dim, *kv_maps, q_map, out_map, p, ctx->num_sms, static_cast<cudaStream_t>(stream)));
        return SW_OK;
    }
    SW_CUDA(sw::launch_mixed_attn(ctx->layout.head_dim, *kv_maps, q_map, out_map, p, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

// Append + attention: one launch, or two where the persistent grid would not be resident at once.
sw_status run_iteration(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, const void* k_new, const void* v_new, const void* q,
                        void* out, float* lse, void* stream, const char* who, Window window = {}) {
    if (ctx && !(window.keys > 0 ? ctx->window_grid_resident : ctx->grid_resident)) {
        sw_status st = sw_kv_append(ctx, kv_pool, batch, k_new, v_new, stream);
        if (st != SW_OK) return st;
        return run_mixed(ctx, kv_pool, batch, nullptr, nullptr, q, out, lse, stream, who, window);
    }
    return run_mixed(ctx, kv_pool, batch, k_new, v_new, q, out, lse, stream, who, window);
}
}  // namespace

sw_status sw_mixed_attn_run(sw_ctx* ctx, const void* kv_pool, const sw_batch* batch, const void* q, void* out, float* lse,
                            void* stream) {
    return run_mixed(ctx, const_cast<void*>(kv_pool), batch, nullptr, nullptr, q, out, lse, stream, "sw_mixed_attn_run");
}

sw_status sw_mixed_iteration_run(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, const void* k_new, const void* v_new,
                                 const void* q, void* out, float* lse, void* stream) {
    if (!k_new || !v_new) return sw_fail(SW_ERR_INVALID_ARG, "sw_mixed_iteration_run: null tensor");
    return run_iteration(ctx, kv_pool, batch, k_new, v_new, q, out, lse, stream, "sw_mixed_iteration_run");
}

// ---- sliding window with sinks ------------------------------------------------------------------------------------
sw_status sw_mixed_attn_window_run(sw_ctx* ctx, const void* kv_pool, const sw_batch* batch, int32_t window, int32_t sinks, const void* q,
                                   void* out, float* lse, void* stream) {
    Window w;
    sw_status st = check_window(window, sinks, "sw_mixed_attn_window_run", &w);
    if (st != SW_OK) return st;
    return run_mixed(ctx, const_cast<void*>(kv_pool), batch, nullptr, nullptr, q, out, lse, stream, "sw_mixed_attn_window_run", w);
}

sw_status sw_mixed_iteration_window_run(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, int32_t window, int32_t sinks, const void* k_new,
                                        const void* v_new, const void* q, void* out, float* lse, void* stream) {
    Window w;
    sw_status st = check_window(window, sinks, "sw_mixed_iteration_window_run", &w);
    if (st != SW_OK) return st;
    if (!k_new || !v_new) return sw_fail(SW_ERR_INVALID_ARG, "sw_mixed_iteration_window_run: null tensor");
    return run_iteration(ctx, kv_pool, batch, k_new, v_new, q, out, lse, stream, "sw_mixed_iteration_window_run", w);
}

// ---- cross attention -------------------------------------------------------------------------------------------------
sw_status sw_cross_attn_run(sw_ctx* ctx, const void* kv_pool, const sw_batch* batch, const void* q, void* out, float* lse, void* stream) {
    const char* who = "sw_cross_attn_run";
    Chunks ch;
    sw_status st = check_batch(ctx, batch, who, &ch, true);
    if (st != SW_OK) return st;
    if (ch.rows + batch->num_decode == 0) return SW_OK;
    if (!kv_pool || !q || !out) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    if (!aligned16(q, out)) return sw_fail(SW_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned", who);
    const sw::KvMaps* kv_maps = nullptr;
    st = kv_map_for(ctx, const_cast<void*>(kv_pool), &kv_maps);
    if (st != SW_OK) return st;
    const sw_layout& l = ctx->layout;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    // The rows of chunks without keys are written here, and the launch sees the other chunks.
    const int64_t heads = l.num_q_heads;
    int kept = 0;
    for (int j = 0; j < ch.n; ++j) {
        if (ch.P[j] == 0) {
            SW_CUDA(sw::launch_keyless_rows(static_cast<__nv_bfloat16*>(out) + ch.row0[j] * heads * l.head_dim, ch.C[j] * heads * l.head_dim,
                                            lse ? lse + ch.row0[j] * heads : nullptr, ch.C[j] * heads, ctx->num_sms, s));
            continue;
        }
        ch.P[kept] = ch.P[j];
        ch.C[kept] = ch.C[j];
        ch.row0[kept] = ch.row0[j];
        ch.page0[kept] = ch.page0[j];
        ++kept;
    }
    if (kept == 0 && batch->num_decode == 0) return SW_OK;
    sw_batch rest = *batch;
    int64_t skipped = 0;
    if (kept < ch.n) {   // (a launch's first chunk begins at its first row and page)
        skipped = kept > 0 ? ch.row0[0] : 0;
        const int pages = kept > 0 ? ch.page0[0] : 0;
        for (int j = 0; j < kept; ++j) {
            ch.row0[j] -= (int)skipped;
            ch.page0[j] -= pages;
        }
        for (int j = kept; j < ch.n; ++j) ch.P[j] = ch.C[j] = ch.row0[j] = 0;
        ch.n = kept;
        ch.rows -= (int)skipped;
        rest.prefill_pages += pages;
        rest.num_prefill_pages -= pages;
        for (int j = kept; j <= sw::kMaxChunks; ++j) ch.page0[j] = rest.num_prefill_pages;
    }
    const sw::MixedParams p = mixed_params(ctx, &rest, ch, static_cast<const __nv_bfloat16*>(q) + skipped * heads * l.head_dim,
                                           static_cast<__nv_bfloat16*>(out) + skipped * heads * l.head_dim, lse ? lse + skipped * heads : nullptr);
    CUtensorMap q_map = kv_maps->half, out_map = kv_maps->half;
    st = encode_row_maps(ctx, p, &q_map, &out_map);
    if (st != SW_OK) return st;
    SW_CUDA(sw::launch_cross_attn(l.head_dim, *kv_maps, q_map, out_map, p, ctx->num_sms, s));
    return SW_OK;
}

// ---- rotary positions ------------------------------------------------------------------------------------------------
namespace {
// Rows of `width` elements, `stride` apart.
struct Rows {
    const void* at;
    int64_t stride, width;
    const char* name;
};
bool rows_overlap(const Rows& a, const Rows& b, int64_t rows) {   // by their extents, as numbers
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.at), b0 = reinterpret_cast<uintptr_t>(b.at);
    const uintptr_t a1 = a0 + (uintptr_t)((rows - 1) * a.stride + a.width) * 2, b1 = b0 + (uintptr_t)((rows - 1) * b.stride + b.width) * 2;
    return a0 < b1 && b0 < a1;
}

// pool: the keys and values go there; null: the keys go to k_out.
sw_status run_rope(sw_ctx* ctx, void* kv_pool, bool append, const sw_batch* batch, const sw_rope* rope, const void* q, const void* k, const void* v,
                   void* q_out, void* k_out, void* stream, const char* who) {
    Chunks ch;
    sw_status st = check_batch(ctx, batch, who, &ch);
    if (st != SW_OK) return st;
    const sw_layout& l = ctx->layout;
    if (!rope || !rope->turns) return sw_fail(SW_ERR_INVALID_ARG, "%s: null rope or frequencies", who);
    if (rope->rotary_dim < 16 || rope->rotary_dim % 16 != 0 || rope->rotary_dim > l.head_dim)
        return sw_fail(SW_ERR_UNSUPPORTED, "%s: rotary_dim %d (multiples of 16 up to the head size, %d)", who, rope->rotary_dim, l.head_dim);
    const int64_t q_width = (int64_t)l.num_q_heads * l.head_dim, kv_width = (int64_t)l.num_kv_heads * l.head_dim;
    const int64_t q_stride = rope->q_stride ? rope->q_stride : q_width, k_stride = rope->k_stride ? rope->k_stride : kv_width,
                  v_stride = append && rope->v_stride ? rope->v_stride : kv_width;   // (ignored where there are no values)
    if (q_stride < q_width || k_stride < kv_width || v_stride < kv_width || ((q_stride | k_stride | v_stride) & 7) != 0 ||
        std::max(q_stride, std::max(k_stride, v_stride)) > (int64_t)1 << 31)   // (times the rows, in bytes, that fits 64 bits)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: strides of %lld, %lld, %lld elements (multiples of 8, a row's width at least)", who, (long long)q_stride,
                       (long long)k_stride, (long long)v_stride);
    const int64_t rows = ch.rows + batch->num_decode;
    if (rows == 0) return SW_OK;
    if (!q || !k || !q_out || (append ? !kv_pool || !v : !k_out)) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    if (!aligned16(q, k, v, q_out) || !aligned16(kv_pool, k_out)) return sw_fail(SW_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned", who);
    if ((reinterpret_cast<uintptr_t>(rope->turns) & 7) != 0) return sw_fail(SW_ERR_INVALID_ARG, "%s: frequencies must be 8-byte aligned", who);
    // A row is read by the warps that write it, so dense rows can be rotated where they are; any other overlap would be read too late.
    const Rows in[] = {{q, q_stride, q_width, "q"}, {k, k_stride, kv_width, "k"}, {v, v_stride, kv_width, "v"}};
    const Rows out[] = {{q_out, q_width, q_width, "q_out"}, {k_out, kv_width, kv_width, "k_out"}};
    for (int o = 0; o < (append ? 1 : 2); ++o)
        for (int i = 0; i < (append ? 3 : 2); ++i)
            if (rows_overlap(out[o], in[i], rows) && !(o == i && out[o].at == in[i].at && out[o].stride == in[i].stride))
                return sw_fail(SW_ERR_INVALID_ARG, "%s: %s overlaps %s", who, out[o].name, in[i].name);
    const int64_t pool_elements = l.num_pages * 2 * l.num_kv_heads * sw::kPageSize * l.head_dim;
    if (append && rows_overlap(out[0], Rows{kv_pool, 0, pool_elements, "the pool"}, rows)) return sw_fail(SW_ERR_INVALID_ARG, "%s: q_out overlaps the pool", who);
    if (!append && rows_overlap(out[0], out[1], rows)) return sw_fail(SW_ERR_INVALID_ARG, "%s: q_out overlaps k_out", who);
    st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    sw::RopeParams p{};
    p.append = append_params(ctx, batch, ch, append ? kv_pool : nullptr, k, v);
    p.Hq = l.num_q_heads;
    p.rotary = rope->rotary_dim;
    p.interleaved = rope->interleaved != 0;
    p.magnitude = rope->magnitude;
    p.turns = rope->turns;
    p.positions = rope->positions;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_out = static_cast<__nv_bfloat16*>(q_out);
    p.k_out = static_cast<__nv_bfloat16*>(k_out);
    SW_CUDA(sw::launch_rope(p, l.head_dim, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}
}  // namespace

sw_status sw_rope_append(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, const sw_rope* rope, const void* q, const void* k_new, const void* v_new,
                         void* q_out, void* stream) {
    return run_rope(ctx, kv_pool, true, batch, rope, q, k_new, v_new, q_out, nullptr, stream, "sw_rope_append");
}

sw_status sw_rope_run(sw_ctx* ctx, const sw_batch* batch, const sw_rope* rope, const void* q, const void* k, void* q_out, void* k_out, void* stream) {
    return run_rope(ctx, nullptr, false, batch, rope, q, k, nullptr, q_out, k_out, stream, "sw_rope_run");
}

// ---- sampling ----------------------------------------------------------------------------------------------------------
sw_status sw_sample_run(sw_ctx* ctx, const sw_sampling* sampling, int32_t* tokens, float* log_probs, void* stream) {
    const char* who = "sw_sample_run";
    if (!ctx || !sampling) return sw_fail(SW_ERR_INVALID_ARG, "%s: null context or sampling", who);
    const sw_sampling& a = *sampling;
    if (a.dtype != SW_DTYPE_F32 && a.dtype != SW_DTYPE_BF16 && a.dtype != SW_DTYPE_F16) return sw_fail(SW_ERR_UNSUPPORTED, "%s: dtype %d", who, a.dtype);
    if (a.rows < 0 || a.vocab < 1 || a.row_stride < a.vocab)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: %d rows of %d logits, %lld apart", who, a.rows, a.vocab, (long long)a.row_stride);
    if (a.vocab > sw::kMaxVocab || a.rows > SW_SAMPLE_MAX_ROWS)
        return sw_fail(SW_ERR_UNSUPPORTED, "%s: %d rows of %d logits (at most %d of %d)", who, a.rows, a.vocab, SW_SAMPLE_MAX_ROWS, sw::kMaxVocab);
    if (a.rows == 0) return SW_OK;
    if (!a.logits || !a.uniform || !tokens) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    if (reinterpret_cast<uintptr_t>(a.logits) % (a.dtype == SW_DTYPE_F32 ? 4 : 2) != 0)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: logits must be aligned to their size", who);
    const sw_status st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    sw::SampleParams p{};
    p.logits = a.logits;
    p.rows = a.rows;
    p.vocab = a.vocab;
    p.row_stride = a.row_stride;
    p.temperature = a.temperature;
    p.top_k = a.top_k;
    p.top_p = a.top_p;
    p.min_p = a.min_p;
    p.uniform = a.uniform;
    p.tokens = tokens;
    p.log_probs = log_probs;
    SW_CUDA(sw::launch_sample(p, a.dtype, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

// ---- the pool in 8 bits --------------------------------------------------------------------------------------------
namespace {
// Pages that the chunks' prompts take in 16 bits, and what they take in bytes with their list.
int64_t prompt_pages(const Chunks& ch) {
    int64_t pages = 0;
    for (int j = 0; j < ch.n; ++j) pages += ((int64_t)ch.P[j] + ch.C[j] + sw::kPageSize - 1) / sw::kPageSize;
    return pages;
}
size_t page_bytes(const sw_layout& l) { return (size_t)2 * l.num_kv_heads * sw::kPageSize * l.head_dim * 2; }
size_t kv8_scratch(const sw_layout& l, int64_t pages) { return (size_t)pages * page_bytes(l) + align_up((size_t)pages * 4, 256); }

// Whether an iteration's chunks read a 16-bit copy of their prompts, made by a launch of its own, rather than the 8-bit pool.  Measured with
// 32/8/128: a 128-key step of an entry is up to 0.9 us longer over the 8-bit pool (the widened V tiles go through a shared memory that the
// tensor cores' operands keep busy), a copy costs 4 us and 0.6 us a megabyte of the prompts, and most of the rest is the same.  Over the
// pool | with a copy, us: 1024 tokens at prefix 4096 104 | 78, 512 at 512 31 | 27, 4096 at 28672 2040 | 1575; 128 at 28672 94 | 110.
bool chunks_copied(const sw_layout& l, const Chunks& ch, int num_sms) {
    const int group = l.num_q_heads / l.num_kv_heads;
    double steps = 0., megabytes = 0.;
    for (int j = 0; j < ch.n; ++j) {
        const double items = ((int64_t)ch.C[j] * group + 255) / 256 * (double)l.num_kv_heads;
        steps += items * (((double)ch.P[j] + 0.5 * ch.C[j]) / 128. + 1.);
        megabytes += ((double)ch.P[j] + ch.C[j]) * 2 * l.num_kv_heads * l.head_dim * 1e-6;
    }
    return 0.9 * steps / num_sms > 1. + 0.6 * megabytes;
}

sw_status kv8_maps_for(sw_ctx* ctx, const void* pool, const sw::KvMaps** out) {
    for (int i = 0; i < ctx->kv8_map_count; ++i)
        if (ctx->kv8_maps[i].pool == pool) {
            *out = &ctx->kv8_maps[i].maps;
            return SW_OK;
        }
    sw_ctx::Kv8MapEntry& e = ctx->kv8_maps[ctx->kv8_map_next];
    e.pool = nullptr;
    CUresult r = sw::encode_kv8_maps(ctx->encode, ctx->layout, pool, &e.maps);
    if (r != CUDA_SUCCESS) return sw_fail(SW_ERR_CUDA, "cuTensorMapEncodeTiled(8-bit pool) failed with CUresult %d", (int)r);
    e.pool = pool;
    constexpr int kMost = sizeof ctx->kv8_maps / sizeof ctx->kv8_maps[0];
    ctx->kv8_map_next = (ctx->kv8_map_next + 1) % kMost;
    ctx->kv8_map_count = std::min(ctx->kv8_map_count + 1, kMost);
    *out = &e.maps;
    return SW_OK;
}
}  // namespace

size_t sw_kv8_scratch_bytes(const sw_layout* layout, int64_t prompt_pages) {
    if (!layout || !layout_supported(*layout) || prompt_pages < 0 || prompt_pages > (int64_t)1 << 30 ||
        2 * prompt_pages * layout->num_kv_heads >= (int64_t)1 << 31)
        return 0;
    return kv8_scratch(*layout, prompt_pages);
}

sw_status sw_kv8_append(sw_ctx* ctx, void* kv8_pool, float* scales, const sw_batch* batch, const void* k_new, const void* v_new, void* stream) {
    Chunks ch;
    sw_status st = check_batch(ctx, batch, "sw_kv8_append", &ch);
    if (st != SW_OK) return st;
    if (ch.rows + batch->num_decode == 0) return SW_OK;
    if (!kv8_pool || !scales || !k_new || !v_new) return sw_fail(SW_ERR_INVALID_ARG, "sw_kv8_append: null tensor");
    st = check_current_device(ctx, "sw_kv8_append");
    if (st != SW_OK) return st;
    if (!aligned16(kv8_pool, k_new, v_new, scales)) return sw_fail(SW_ERR_INVALID_ARG, "sw_kv8_append: tensors must be 16-byte aligned");
    const sw::AppendParams p = append_params(ctx, batch, ch, nullptr, k_new, v_new);
    SW_CUDA(sw::launch_kv8_append(p, ch.C, static_cast<uint8_t*>(kv8_pool), scales, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

sw_status sw_kv8_attn_run(sw_ctx* ctx, const void* kv8_pool, const float* scales, const sw_batch* batch, const void* q, void* out, float* lse,
                          void* scratch, size_t scratch_bytes, void* stream) {
    const char* who = "sw_kv8_attn_run";
    Chunks ch;
    sw_status st = check_batch(ctx, batch, who, &ch);
    if (st != SW_OK) return st;
    if (ch.rows + batch->num_decode == 0) return SW_OK;
    if (!kv8_pool || !scales || !q || !out) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    if (!aligned16(kv8_pool, q, out, scales)) return sw_fail(SW_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned", who);
    const sw_layout& l = ctx->layout;
    const sw::KvMaps* maps = nullptr;
    st = kv8_maps_for(ctx, kv8_pool, &maps);
    if (st != SW_OK) return st;
    sw::MixedParams p = mixed_params(ctx, batch, ch, q, out, lse);
    p.kv8_scales = scales;
    // Pages are half as long, but a warp needs two thirds of the time for one: 64 contexts of 256-2048 tokens beside 512 at prefix 512 take
    // 70 us with the half, 59 with three quarters, 61 with the whole; 128 log-normal ones beside 1024 at 4096 274, 262 and 277.
    p.stage_us *= 0.75f;
    p.stages_per_us *= 4.f / 3.f;
    p.steps_per_stage *= 0.75f;
    CUtensorMap q_map = maps->half, out_map = maps->half;
    st = encode_row_maps(ctx, p, &q_map, &out_map);
    if (st != SW_OK) return st;
    const int64_t pages = prompt_pages(ch);
    if (scratch && (reinterpret_cast<uintptr_t>(scratch) & 255) != 0)
        return sw_fail(SW_ERR_WORKSPACE, "%s: scratch must be 256-byte aligned", who);
    if (scratch && pages > 0 && pages <= (int64_t)1 << 30 && 2 * pages * l.num_kv_heads < (int64_t)1 << 31 &&
        scratch_bytes >= kv8_scratch(l, pages) && chunks_copied(l, ch, ctx->num_sms)) {
        __nv_bfloat16* copy = static_cast<__nv_bfloat16*>(scratch);
        int32_t* list = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(scratch) + (size_t)pages * page_bytes(l));
        sw_layout copy_layout = l;
        copy_layout.num_pages = pages;
        sw::KvMaps copy_maps;
        CUresult r = sw::encode_kv_maps(ctx->encode, copy_layout, copy, &copy_maps);
        if (r != CUDA_SUCCESS) return sw_fail(SW_ERR_CUDA, "cuTensorMapEncodeTiled(scratch) failed with CUresult %d", (int)r);
        copy_maps.page = maps->page;
        SW_CUDA(sw::launch_kv8_expand(append_params(ctx, batch, ch, nullptr, nullptr, nullptr), ch.C, static_cast<const uint8_t*>(kv8_pool), scales,
                                      copy, list, ctx->num_sms, static_cast<cudaStream_t>(stream)));
        p.prefill_pages = list;
        p.num_prefill_pages = (int)pages;
        p.chunk_pool_pages = pages;
        for (int j = 0; j < sw::kMaxChunks; ++j)
            p.cPage0[j + 1] = p.cPage0[j] + (j < ch.n ? (int)(((int64_t)ch.P[j] + ch.C[j] + sw::kPageSize - 1) / sw::kPageSize) : 0);
        SW_CUDA(sw::launch_kv8_attn(l.head_dim, true, copy_maps, q_map, out_map, p, ctx->num_sms, static_cast<cudaStream_t>(stream)));
        return SW_OK;
    }
    SW_CUDA(sw::launch_kv8_attn(l.head_dim, false, *maps, q_map, out_map, p, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

// ---- weights of keys, and eviction by them ---------------------------------------------------------------------------
namespace {
size_t score_bytes_per_page(const sw_layout& l) { return (size_t)sw::kPageSize * l.num_q_heads * 4; }
sw_status check_weights(const sw_key_weights* w, const char* who) {
    if (!w || !w->weights || !w->row_of) return sw_fail(SW_ERR_INVALID_ARG, "%s: null weights or rows", who);
    if (w->rows < 1 || w->capacity < 1) return sw_fail(SW_ERR_INVALID_ARG, "%s: %lld rows of %d weights", who, (long long)w->rows, w->capacity);
    return SW_OK;
}
// The CTAs of an eviction read the batch's and the lists' words while others already write what it returns (lengths updated in place would be read as
// old ones by some of a request's CTAs and as new ones by others, which wait for one another).  The page lists' own lengths are on the device.
sw_status check_evict_arrays(const sw_batch* b, const sw_key_weights* w, int num_kv_heads, const int32_t* new_page_indptr, const int32_t* new_pages,
                             const int32_t* new_row_of, int32_t budget, const int32_t* kept, const int32_t* new_len, const char* who) {
    struct Words {
        const int32_t* at;
        int64_t count;
        const char* name;
    };
    const int64_t n = b->num_decode;
    const Words out[2] = {{new_len, n, "new_len"}, {kept, n * num_kv_heads * std::max(budget, 1), "kept"}};
    const Words in[] = {{b->decode_kv_len, n, "decode_kv_len"}, {b->decode_page_indptr, n + 1, "decode_page_indptr"}, {b->decode_pages, 1, "decode_pages"},
                        {w ? w->row_of : nullptr, n, "row_of"}, {new_page_indptr, n + 1, "new_page_indptr"}, {new_pages, 1, "new_pages"},
                        {new_row_of, n, "new_row_of"}, out[0]};
    auto overlap = [](const Words& a, const Words& c) {   // (as numbers: the arrays need not be parts of one)
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.at), c0 = reinterpret_cast<uintptr_t>(c.at);
        return a.at && c.at && a0 < c0 + (uintptr_t)c.count * 4 && c0 < a0 + (uintptr_t)a.count * 4;
    };
    for (const Words& o : out)
        for (const Words& i : in)
            if (o.name != i.name && overlap(o, i)) return sw_fail(SW_ERR_INVALID_ARG, "%s: %s overlaps %s", who, o.name, i.name);
    return SW_OK;
}
}  // namespace

size_t sw_attn_weights_scratch_bytes(const sw_layout* layout, int64_t decode_pages) {
    if (!layout || !layout_supported(*layout) || decode_pages < 0 || decode_pages > INT32_MAX) return 0;
    return (size_t)decode_pages * score_bytes_per_page(*layout);
}

sw_status sw_decode_attn_weights_run(sw_ctx* ctx, const void* kv_pool, const sw_batch* batch, const void* q, void* out, float* lse,
                                     const sw_key_weights* weights, void* scratch, size_t scratch_bytes, void* stream) {
    const char* who = "sw_decode_attn_weights_run";
    Chunks ch;
    sw_status st = check_batch(ctx, batch, who, &ch);
    if (st != SW_OK) return st;
    if (ch.rows > 0) return sw_fail(SW_ERR_UNSUPPORTED, "%s: decode-only (no chunks)", who);
    if (batch->num_decode == 0) return SW_OK;
    if (!kv_pool || !q || !out || !lse || !scratch) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    st = check_weights(weights, who);
    if (st != SW_OK) return st;
    st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    if (!aligned16(q, out, lse)) return sw_fail(SW_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned", who);
    if ((reinterpret_cast<uintptr_t>(scratch) & 127) != 0) return sw_fail(SW_ERR_WORKSPACE, "%s: scratch must be 128-byte aligned", who);
    const sw::KvMaps* kv_maps = nullptr;
    st = kv_map_for(ctx, kv_pool, &kv_maps);
    if (st != SW_OK) return st;
    const sw_layout& l = ctx->layout;
    sw::MixedParams p = mixed_params(ctx, batch, ch, q, out, lse);
    p.scores = static_cast<float*>(scratch);
    p.score_pages = (int64_t)(scratch_bytes / score_bytes_per_page(l));
    sw::WeightParams w{};
    w.n = p.n;
    w.Hkv = p.Hkv;
    w.group = p.group;
    w.capacity = weights->capacity;
    w.rows = weights->rows;
    w.kv_len = p.decode_kv_len;
    w.page_indptr = p.decode_page_indptr;
    w.row_of = weights->row_of;
    w.scores = p.scores;
    w.lse = lse;
    w.score_pages = p.score_pages;
    w.weights = weights->weights;
    w.ctrl = p.ctrl;
    SW_CUDA(sw::launch_scored_attn(l.head_dim, *kv_maps, kv_maps->half, p, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    SW_CUDA(sw::launch_key_weights(w, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

sw_status sw_kv_evict(sw_ctx* ctx, void* kv_pool, const sw_batch* batch, const sw_key_weights* weights, const int32_t* new_page_indptr,
                      const int32_t* new_pages, const int32_t* new_row_of, int32_t budget, int32_t sinks, int32_t recent, int32_t* kept,
                      int32_t* new_len, void* stream) {
    const char* who = "sw_kv_evict";
    Chunks ch;
    sw_status st = SW_OK;
    if (batch && (batch->chunk_len > 0 || batch->num_chunks > 0)) return sw_fail(SW_ERR_UNSUPPORTED, "%s: decode requests only (no chunks)", who);
    if (batch && batch->num_decode > 0)
        st = check_evict_arrays(batch, weights, ctx ? ctx->layout.num_kv_heads : 1, new_page_indptr, new_pages, new_row_of, budget, kept, new_len, who);
    if (st == SW_OK) st = check_batch(ctx, batch, who, &ch);
    if (st != SW_OK) return st;
    if (batch->num_decode == 0) return SW_OK;
    if (!kv_pool || !new_page_indptr || !new_pages || !new_row_of || !kept || !new_len) return sw_fail(SW_ERR_INVALID_ARG, "%s: null tensor", who);
    st = check_weights(weights, who);
    if (st != SW_OK) return st;
    if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget || budget > weights->capacity)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: budget %d (sinks %d, recent %d, capacity %d)", who, budget, sinks, recent, weights->capacity);
    st = check_current_device(ctx, who);
    if (st != SW_OK) return st;
    if (!aligned16(kv_pool)) return sw_fail(SW_ERR_INVALID_ARG, "%s: kv_pool must be 16-byte aligned", who);
    sw::EvictParams p{};
    p.n = batch->num_decode;
    p.Hkv = ctx->layout.num_kv_heads;
    p.capacity = weights->capacity;
    p.budget = budget;
    p.sinks = sinks;
    p.recent = recent;
    p.num_pages = ctx->layout.num_pages;
    p.rows = weights->rows;
    p.kv_len = batch->decode_kv_len;
    p.page_indptr = batch->decode_page_indptr;
    p.pages = batch->decode_pages;
    p.row_of = weights->row_of;
    p.new_page_indptr = new_page_indptr;
    p.new_pages = new_pages;
    p.new_row_of = new_row_of;
    p.weights = weights->weights;
    p.pool = static_cast<__nv_bfloat16*>(kv_pool);
    p.kept = kept;
    p.new_len = new_len;
    p.ctrl = reinterpret_cast<int32_t*>(ctx->ws + ctx->w.ctrl);
    SW_CUDA(sw::launch_evict(p, ctx->layout.head_dim, ctx->num_sms, static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

namespace {
// The device copies of a host batch's page tables, inside the workspace.
struct HostTables {
    int32_t *len, *indptr, *dec_pages, *pf_pages;
};

sw_status copy_tables(const sw_batch* hb, const HostTables& t, int64_t n_dec_pages, cudaStream_t s) {
    const int n = hb->num_decode;
    if (n > 0) {
        SW_CUDA(cudaMemcpyAsync(t.len, hb->decode_kv_len, (size_t)n * 4, cudaMemcpyHostToDevice, s));
        SW_CUDA(cudaMemcpyAsync(t.indptr, hb->decode_page_indptr, (size_t)(n + 1) * 4, cudaMemcpyHostToDevice, s));
        if (n_dec_pages > 0)
            SW_CUDA(cudaMemcpyAsync(t.dec_pages, hb->decode_pages, (size_t)n_dec_pages * 4, cudaMemcpyHostToDevice, s));
    }
    if (hb->num_prefill_pages > 0)
        SW_CUDA(cudaMemcpyAsync(t.pf_pages, hb->prefill_pages, (size_t)hb->num_prefill_pages * 4, cudaMemcpyHostToDevice, s));
    return SW_OK;
}

// Whether two parts of the iteration would meet on a page: one that rows of two chunks are written to (tokens of one prompt, say; the
// second chunk may attend the first one's rows of that page), or chunk rows and a decode request's last row.  Such an iteration is not
// taken apart, since every row is written before anything is attended.
bool parts_share_a_page(const sw_batch* hb, const Chunks& ch) {
    std::vector<int32_t> written;
    for (int j = 0; j < ch.n; ++j)
        for (int64_t pi = ch.P[j] / sw::kPageSize; pi <= ((int64_t)ch.P[j] + ch.C[j] - 1) / sw::kPageSize; ++pi)
            written.push_back(hb->prefill_pages[ch.page0[j] + pi]);
    std::sort(written.begin(), written.end());
    if (std::adjacent_find(written.begin(), written.end()) != written.end()) return true;
    for (int i = 0; i < hb->num_decode; ++i) {
        const int pages = (int)(((int64_t)hb->decode_kv_len[i] + sw::kPageSize - 1) / sw::kPageSize);
        const int beg = hb->decode_page_indptr[i], end = hb->decode_page_indptr[i + 1];
        if (pages < 1 || beg < 0 || end > hb->decode_page_indptr[hb->num_decode] || pages > end - beg) continue;
        if (std::binary_search(written.begin(), written.end(), hb->decode_pages[beg + pages - 1])) return true;
    }
    return false;
}

// Chunk rows of a part of a host-buffer iteration (0: it is run whole).  Parts are whole 256-row groups.  Where the chunks'
// arithmetic (at 1.2 PFLOP/s) takes longer than the way up (at 46 GB/s), parts of fewer work items than there are SMs would cost
// more than they hide.
int host_part_rows(const sw_layout& l, int num_sms, const sw_batch* hb, const Chunks& ch) {
    const size_t up_bytes = ((size_t)ch.rows + hb->num_decode) * (l.num_q_heads + 2 * l.num_kv_heads) * l.head_dim * 2;
    if (ch.rows == 0 || up_bytes < kHostPartBytes) return 0;
    const int group_rows = 256 / (l.num_q_heads / l.num_kv_heads);
    int groups = ((ch.rows + kHostParts - 1) / kHostParts + group_rows - 1) / group_rows;
    double pairs = 0.;   // attended (query, key) pairs
    for (int j = 0; j < ch.n; ++j) pairs += (double)ch.C[j] * ((double)ch.P[j] + 0.5 * (double)ch.C[j]);
    if (pairs * 4. * l.num_q_heads * l.head_dim / 1.2e15 > (double)up_bytes / 46e9)
        groups = std::max(groups, num_sms / l.num_kv_heads);
    if (groups * group_rows >= ch.rows) return 0;
    try {
        return parts_share_a_page(hb, ch) ? 0 : groups * group_rows;
    } catch (...) {
        return 0;   // no host memory for the comparison
    }
}

// The host-buffer iteration in parts: the decode rows, then the chunk rows in runs of `per` consecutive rows (a chunk cut at a row
// is the same attention: the rows behind the cut have a longer prefix).  While a part computes, the next one's inputs are on their way.
sw_status iterate_parts(sw_ctx* ctx, void* kv_pool, const sw_batch* hb, const Chunks& ch, int per, const HostTables& t,
                        int64_t n_dec_pages, const void* h_q, const void* h_k, const void* h_v, void* h_out, float* h_lse,
                        cudaStream_t s) {
    const sw_layout& l = ctx->layout;
    const size_t q_row = (size_t)l.num_q_heads * l.head_dim * 2, kv_row = (size_t)l.num_kv_heads * l.head_dim * 2;
    uint8_t *d_q = ctx->ws + ctx->w.st_q, *d_k = ctx->ws + ctx->w.st_k, *d_v = ctx->ws + ctx->w.st_v, *d_out = ctx->ws + ctx->w.st_out;
    float* d_lse = h_lse ? reinterpret_cast<float*>(ctx->ws + ctx->w.st_lse) : nullptr;
    const int n = hb->num_decode;
    auto up_rows = [&](int r0, int rows) -> sw_status {
        SW_CUDA(cudaMemcpyAsync(d_k + r0 * kv_row, (const uint8_t*)h_k + r0 * kv_row, rows * kv_row, cudaMemcpyHostToDevice, ctx->copies));
        SW_CUDA(cudaMemcpyAsync(d_v + r0 * kv_row, (const uint8_t*)h_v + r0 * kv_row, rows * kv_row, cudaMemcpyHostToDevice, ctx->copies));
        SW_CUDA(cudaMemcpyAsync(d_q + r0 * q_row, (const uint8_t*)h_q + r0 * q_row, rows * q_row, cudaMemcpyHostToDevice, ctx->copies));
        return SW_OK;
    };
    auto down_rows = [&](int r0, int rows) -> sw_status {
        SW_CUDA(cudaMemcpyAsync((uint8_t*)h_out + r0 * q_row, d_out + r0 * q_row, rows * q_row, cudaMemcpyDeviceToHost, ctx->copies));
        if (h_lse)
            SW_CUDA(cudaMemcpyAsync(h_lse + (size_t)r0 * l.num_q_heads, d_lse + (size_t)r0 * l.num_q_heads,
                                    (size_t)rows * l.num_q_heads * 4, cudaMemcpyDeviceToHost, ctx->copies));
        return SW_OK;
    };
    // the copies come after whatever the caller's stream was doing (it may produce the host buffers)
    SW_CUDA(cudaEventRecord(ctx->ev_start, s));
    SW_CUDA(cudaStreamWaitEvent(ctx->copies, ctx->ev_start, 0));
    sw_status st = copy_tables(hb, t, n_dec_pages, ctx->copies);
    if (st != SW_OK) return st;
    sw_batch part = *hb;
    part.decode_kv_len = t.len;
    part.decode_page_indptr = t.indptr;
    part.decode_pages = t.dec_pages;
    if (n > 0) {
        if ((st = up_rows(ch.rows, n)) != SW_OK) return st;
        SW_CUDA(cudaEventRecord(ctx->ev_up, ctx->copies));
        SW_CUDA(cudaStreamWaitEvent(s, ctx->ev_up, 0));
        part.num_chunks = part.prefix_len = part.chunk_len = part.num_prefill_pages = 0;
        st = sw_mixed_iteration_run(ctx, kv_pool, &part, d_k + ch.rows * kv_row, d_v + ch.rows * kv_row, d_q + ch.rows * q_row,
                                    d_out + ch.rows * q_row, d_lse ? d_lse + (size_t)ch.rows * l.num_q_heads : nullptr, s);
        if (st != SW_OK) return st;
        SW_CUDA(cudaEventRecord(ctx->ev_done[kHostParts], s));
    }
    int done = 0;
    for (int r0 = 0; r0 < ch.rows; r0 += per, ++done) {
        const int rows = std::min(per, ch.rows - r0);
        if ((st = up_rows(r0, rows)) != SW_OK) return st;
        SW_CUDA(cudaEventRecord(ctx->ev_up, ctx->copies));
        SW_CUDA(cudaStreamWaitEvent(s, ctx->ev_up, 0));
        part.num_decode = 0;
        int32_t prefix[sw::kMaxChunks], len[sw::kMaxChunks], pages[sw::kMaxChunks + 1];
        int m = 0, page0 = 0;
        for (int j = 0; j < ch.n; ++j) {
            const int a = std::max(r0, ch.row0[j]), b = std::min(r0 + rows, ch.row0[j] + ch.C[j]);
            if (a >= b) continue;
            if (m == 0) page0 = ch.page0[j];
            prefix[m] = ch.P[j] + (a - ch.row0[j]);
            len[m] = b - a;
            pages[m] = ch.page0[j] - page0;
            pages[++m] = ch.page0[j + 1] - page0;
        }
        part.prefill_pages = t.pf_pages + page0;
        part.num_prefill_pages = pages[m];
        part.num_chunks = m > 1 ? m : 0;
        part.prefix_len = prefix[0];
        part.chunk_len = m > 1 ? rows : len[0];
        part.chunk_prefix_lens = prefix;
        part.chunk_lens = len;
        part.chunk_page_indptr = pages;
        st = sw_mixed_iteration_run(ctx, kv_pool, &part, d_k + r0 * kv_row, d_v + r0 * kv_row, d_q + r0 * q_row, d_out + r0 * q_row,
                                    d_lse ? d_lse + (size_t)r0 * l.num_q_heads : nullptr, s);
        if (st != SW_OK) return st;
        SW_CUDA(cudaEventRecord(ctx->ev_done[done], s));
    }
    // The results follow the last inputs on the same stream: copies of a few megabytes in both directions at once are slower on
    // this platform than one after the other (4 MB each way: 80 us alone, 370 us together).
    if (n > 0) {
        SW_CUDA(cudaStreamWaitEvent(ctx->copies, ctx->ev_done[kHostParts], 0));
        if ((st = down_rows(ch.rows, n)) != SW_OK) return st;
    }
    for (int i = 0; i < done; ++i) {
        SW_CUDA(cudaStreamWaitEvent(ctx->copies, ctx->ev_done[i], 0));
        if ((st = down_rows(i * per, std::min(per, ch.rows - i * per))) != SW_OK) return st;
    }
    return SW_OK;
}
}  // namespace

sw_status sw_mixed_iteration_host(sw_ctx* ctx, void* kv_pool, const sw_batch* hb, const void* h_q, const void* h_k_new,
                                  const void* h_v_new, void* h_out, float* h_lse, void* stream) {
    sw_status st = SW_OK;
    if (!ctx || !hb) return sw_fail(SW_ERR_INVALID_ARG, "sw_mixed_iteration_host: null context or batch");
    Chunks hch;
    st = chunks_of(hb, "sw_mixed_iteration_host", &hch);
    if (st != SW_OK) return st;
    if (hb->chunk_len < 0 || hb->num_decode < 0 || hb->num_prefill_pages < 0 || hch.rows > ctx->max_chunk ||
        hb->num_decode > ctx->max_decode)
        return sw_fail(SW_ERR_WORKSPACE, "sw_mixed_iteration_host: batch exceeds the context's limits");
    const int rows = hch.rows + hb->num_decode;
    if (rows == 0) return SW_OK;
    if (!h_q || !h_k_new || !h_v_new || !h_out || !kv_pool)
        return sw_fail(SW_ERR_INVALID_ARG, "sw_mixed_iteration_host: null tensor");
    const int n = hb->num_decode;
    if (n > 0 && (!hb->decode_kv_len || !hb->decode_page_indptr || !hb->decode_pages))
        return sw_fail(SW_ERR_INVALID_ARG, "sw_mixed_iteration_host: decode arrays missing");
    if (hb->num_prefill_pages > 0 && !hb->prefill_pages)   // (the lists are also read here, see parts_share_a_page)
        return sw_fail(SW_ERR_INVALID_ARG, "sw_mixed_iteration_host: prefill page list missing");
    const int64_t n_dec_pages = n > 0 ? hb->decode_page_indptr[n] : 0;
    if (n_dec_pages < 0 || n_dec_pages + hb->num_prefill_pages > ctx->max_pages)
        return sw_fail(SW_ERR_WORKSPACE, "sw_mixed_iteration_host: %lld page-table entries exceed max_pages %lld",
                       (long long)(n_dec_pages + hb->num_prefill_pages), (long long)ctx->max_pages);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const sw_layout& l = ctx->layout;
    const size_t q_bytes = (size_t)rows * l.num_q_heads * l.head_dim * 2;
    const size_t kv_bytes = (size_t)rows * l.num_kv_heads * l.head_dim * 2;
    uint8_t* ws = ctx->ws;
    int32_t* d_pages = reinterpret_cast<int32_t*>(ws + ctx->w.st_pages);
    HostTables t;                                     // [n], [n+1], then the page lists
    t.len = d_pages;
    t.indptr = t.len + ctx->max_decode;
    t.dec_pages = t.indptr + ctx->max_decode + 2;
    t.pf_pages = t.dec_pages + n_dec_pages;
    sw_batch db = *hb;
    db.prefill_pages = t.pf_pages;
    db.decode_kv_len = t.len;
    db.decode_page_indptr = t.indptr;
    db.decode_pages = t.dec_pages;
    Chunks checked;
    if (check_batch(ctx, &db, "sw_mixed_iteration_run", &checked) == SW_OK && check_current_device(ctx, "sw_mixed_iteration_run") == SW_OK) {
        const int per = host_part_rows(ctx->layout, ctx->num_sms, hb, hch);
        if (per > 0 && ctx->copies) {
            st = iterate_parts(ctx, kv_pool, hb, hch, per, t, n_dec_pages, h_q, h_k_new, h_v_new, h_out, h_lse, s);
            // (after an error too: nothing may still be reading or writing the caller's buffers)
            const cudaError_t e[2] = {cudaStreamSynchronize(s), cudaStreamSynchronize(ctx->copies)};
            if (st != SW_OK) return st;
            for (cudaError_t x : e) SW_CUDA(x);
            return SW_OK;
        }
    }
    SW_CUDA(cudaMemcpyAsync(ws + ctx->w.st_q, h_q, q_bytes, cudaMemcpyHostToDevice, s));
    SW_CUDA(cudaMemcpyAsync(ws + ctx->w.st_k, h_k_new, kv_bytes, cudaMemcpyHostToDevice, s));
    SW_CUDA(cudaMemcpyAsync(ws + ctx->w.st_v, h_v_new, kv_bytes, cudaMemcpyHostToDevice, s));
    st = copy_tables(hb, t, n_dec_pages, s);
    if (st != SW_OK) return st;
    float* d_lse = h_lse ? reinterpret_cast<float*>(ws + ctx->w.st_lse) : nullptr;
    st = sw_mixed_iteration_run(ctx, kv_pool, &db, ws + ctx->w.st_k, ws + ctx->w.st_v, ws + ctx->w.st_q, ws + ctx->w.st_out,
                                d_lse, stream);
    if (st != SW_OK) return st;
    SW_CUDA(cudaMemcpyAsync(h_out, ws + ctx->w.st_out, q_bytes, cudaMemcpyDeviceToHost, s));
    if (h_lse) SW_CUDA(cudaMemcpyAsync(h_lse, d_lse, (size_t)rows * l.num_q_heads * 4, cudaMemcpyDeviceToHost, s));
    SW_CUDA(cudaStreamSynchronize(s));
    return SW_OK;
}

int sw_host_part_rows_of(const sw_layout* layout, int32_t num_sms, const sw_batch* hb) {
    Chunks ch;
    if (!layout || !hb || !layout_supported(*layout) || chunks_of(hb, "sw_host_part_rows_of", &ch) != SW_OK) return -1;
    return host_part_rows(*layout, num_sms, hb, ch);
}

int sw_ctx_set_line_wait(sw_ctx* ctx, int64_t cycles) {
    if (!ctx || cycles < 0 || cycles > sw::kLineWaitCycles) return SW_ERR_INVALID_ARG;
    ctx->line_wait_cycles = cycles;
    return SW_OK;
}

namespace {
// Times iterations of `layers` launches each: attention alone, or (k_new / v_new given) append + attention in one launch.
sw_status probe(sw_ctx* ctx, void* const* kv_pools, int32_t layers, const sw_batch* batch, const void* k_new,
                const void* v_new, const void* q, void* out, int32_t warmup, int32_t reps, int64_t* p50_ns, int64_t* p99_ns,
                int64_t* samples_ns, void* stream, const char* who) {
    if (!ctx || !kv_pools || layers < 1 || reps < 1 || warmup < 0 || !p50_ns || !p99_ns)
        return sw_fail(SW_ERR_INVALID_ARG, "%s: invalid argument", who);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!ctx->ev0) SW_CUDA(cudaEventCreate(&ctx->ev0));
    if (!ctx->ev1) SW_CUDA(cudaEventCreate(&ctx->ev1));
    std::vector<int64_t> t((size_t)reps);
    for (int r = -warmup; r < reps; ++r) {
        SW_CUDA(cudaEventRecord(ctx->ev0, s));
        for (int layer = 0; layer < layers; ++layer) {
            sw_status st = k_new ? run_iteration(ctx, kv_pools[layer], batch, k_new, v_new, q, out, nullptr, stream, who)
                                 : run_mixed(ctx, kv_pools[layer], batch, nullptr, nullptr, q, out, nullptr, stream, who);
            if (st != SW_OK) return st;
        }
        SW_CUDA(cudaEventRecord(ctx->ev1, s));
        SW_CUDA(cudaEventSynchronize(ctx->ev1));
        float ms = 0.f;
        SW_CUDA(cudaEventElapsedTime(&ms, ctx->ev0, ctx->ev1));
        if (r >= 0) t[(size_t)r] = (int64_t)std::llround((double)ms * 1e6);
    }
    if (samples_ns) std::memcpy(samples_ns, t.data(), sizeof(int64_t) * (size_t)reps);
    std::sort(t.begin(), t.end());
    // nearest-rank percentiles: the ceil(q * reps)-th smallest sample
    auto rank = [&](double qv) { return t[(size_t)std::max<int64_t>(1, (int64_t)std::ceil(qv * reps)) - 1]; };
    *p50_ns = rank(0.50);
    *p99_ns = rank(0.99);
    return SW_OK;
}
}  // namespace

sw_status sw_cost_probe(sw_ctx* ctx, void* const* kv_pools, int32_t layers, const sw_batch* batch, const void* q, void* out,
                        int32_t warmup, int32_t reps, int64_t* p50_ns, int64_t* p99_ns, int64_t* samples_ns, void* stream) {
    return probe(ctx, kv_pools, layers, batch, nullptr, nullptr, q, out, warmup, reps, p50_ns, p99_ns, samples_ns, stream,
                 "sw_cost_probe");
}

sw_status sw_cost_probe_iteration(sw_ctx* ctx, void* const* kv_pools, int32_t layers, const sw_batch* batch, const void* k_new,
                                  const void* v_new, const void* q, void* out, int32_t warmup, int32_t reps, int64_t* p50_ns,
                                  int64_t* p99_ns, int64_t* samples_ns, void* stream) {
    if (!k_new || !v_new) return sw_fail(SW_ERR_INVALID_ARG, "sw_cost_probe_iteration: null tensor");
    return probe(ctx, kv_pools, layers, batch, k_new, v_new, q, out, warmup, reps, p50_ns, p99_ns, samples_ns, stream,
                 "sw_cost_probe_iteration");
}

sw_status sw_check_status(sw_ctx* ctx, void* stream, int32_t* code, int32_t* detail) {
    if (!ctx) return sw_fail(SW_ERR_INVALID_ARG, "sw_check_status: null context");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int32_t words[2] = {0, 0};
    int32_t* d = reinterpret_cast<int32_t*>(ctx->ws + ctx->w.ctrl) + sw::kCtrStatus;
    SW_CUDA(cudaMemcpyAsync(words, d, sizeof words, cudaMemcpyDeviceToHost, s));
    SW_CUDA(cudaStreamSynchronize(s));
    if (words[0] != 0) {
        // A launch that reported a problem may have skipped units or left early, so the work counters and tickets
        // may not have been re-armed: clear them together with the status words (the stream is idle here).
        SW_CUDA(cudaMemsetAsync(ctx->ws + ctx->w.ctrl, 0, ctx->w.part_ml - ctx->w.ctrl, s));
        SW_CUDA(cudaMemsetAsync(ctx->ws + ctx->w.pf_tickets, 0, ctx->w.pf_ml - ctx->w.pf_tickets, s));
        SW_CUDA(cudaStreamSynchronize(s));
    }
    if (code) *code = words[0];
    if (detail) *detail = words[1];
    if (words[0] != 0)
        return sw_fail((sw_status)words[0], "device reported status %d at site %d index %d", words[0], (words[1] >> 24) & 0xFF,
                       words[1] & 0xFFFFFF);
    return SW_OK;
}

sw_status sw_selftest_wait_timeout(sw_ctx* ctx, int64_t budget_cycles, void* stream) {
    if (!ctx || budget_cycles < 0 || budget_cycles > 4000000000LL)
        return sw_fail(SW_ERR_INVALID_ARG, "sw_selftest_wait_timeout: invalid argument (budget of at most 4e9 cycles)");
    SW_CUDA(sw::launch_selftest_wait(reinterpret_cast<int32_t*>(ctx->ws + ctx->w.ctrl), (long long)budget_cycles,
                                     static_cast<cudaStream_t>(stream)));
    return SW_OK;
}

}  // extern "C"
