// C ABI of libspdp (declared in spdp.h): argument checks, handle life cycle, host-side layout
// of the split-K work partition.  Every numerical step runs in the kernels of pack.cu and
// spmspv.cu.
#include <cuda.h>

#include <cstdio>
#include <cstring>
#include <new>

#include "spdp_hostdev.h"
#include "spdp_internal.h"

namespace spdp {

static thread_local char g_cuda_error[256] = "";

void note_cuda_error(cudaError_t e, const char* what) {
    std::snprintf(g_cuda_error, sizeof(g_cuda_error), "%s: %s (%s)", what, cudaGetErrorName(e),
                  cudaGetErrorString(e));
    cudaGetLastError();   // clear the sticky-free error state
}

namespace {

// Makes `device` current for a scope.
struct DeviceScope {
    int before = -1;
    explicit DeviceScope(int device) {
        if (cudaGetDevice(&before) != cudaSuccess || before == device || cudaSetDevice(device) != cudaSuccess) before = -1;
    }
    ~DeviceScope() {
        if (before >= 0) cudaSetDevice(before);
    }
};

void drop_host_graph(spdp_matrix* h) {
    if (h->host_exec != nullptr) cudaGraphExecDestroy(h->host_exec);
    if (h->host_graph != nullptr) cudaGraphDestroy(h->host_graph);
    h->host_exec = nullptr;
    h->host_graph = nullptr;
}

void release(spdp_matrix* h) {
    if (h == nullptr) return;
    {
        DeviceScope on(h->device);
        // the handle's memory may be in use on any stream (cudaFree would wait for them too)
        const bool idle = cudaDeviceSynchronize() == cudaSuccess;
        for (DeviceBlock* b : {&h->arrays, &h->values_block, &h->workspace_block, &h->packing}) handle_give(h->device, *b, idle);
        if (!idle) cudaGetLastError();
        cudaFree(h->probe_items);
        cudaFree(h->probe_count);
        drop_host_graph(h);
        if (h->capture_stream != nullptr) cudaStreamDestroy(h->capture_stream);
    }
    count_handle(h->device, -1);
    h->magic = 0;
    delete h;
}

spdp_status new_handle(int64_t M, int64_t K, int pad_elems, spdp_matrix** out) {
    if (M < 1 || K < 1 || M > (int64_t(1) << 30) || K > (int64_t(1) << 30)) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (pad_elems != 8 && pad_elems != 1 && pad_elems != 32) return SPDP_ERR_UNSUPPORTED_SHAPE;
    spdp_matrix* h = new (std::nothrow) spdp_matrix();
    if (h == nullptr) return SPDP_ERR_ALLOC;
    std::memset(h, 0, sizeof(*h));
    h->magic = kMagic;
    h->M = M;
    h->K = K;
    h->R = (M + kTileM - 1) / kTileM;
    h->C = (K + kTileK - 1) / kTileK;
    h->NGT = h->R * h->C;
    h->pad_elems = pad_elems;
    // the kernel packs a column-tile index and a 6-bit count into 32 bits
    if (h->NGT * kTileK >= (int64_t(1) << 26)) { delete h; return SPDP_ERR_UNSUPPORTED_SHAPE; }
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, h->device);
    if (e != cudaSuccess) { note_cuda_error(e, "device query"); delete h; return SPDP_ERR_CUDA; }
    count_handle(h->device, 1);
    *out = h;
    return SPDP_OK;
}

// Allocates the arrays whose sizes follow from the shape (on `s`), as one piece.
spdp_status alloc_arrays(spdp_matrix* h, cudaStream_t s) {
    const int64_t cols = h->NGT * kTileK;
    size_t at = 0;
    auto place = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const size_t bitmap = place(cols * kWordsPerCol * sizeof(uint64_t)), colinfo = place(cols * sizeof(uint32_t)),
                 tileoffset = place((h->NGT + 1) * sizeof(uint32_t)), scales = place(h->q4 ? cols * sizeof(__half) : 0),
                 x = place(h->K * sizeof(__half)), mask = place((h->K + 31) / 32 * sizeof(uint32_t)), y = place(h->M * sizeof(float)),
                 status = place(2 * sizeof(int) + kPackTotals * sizeof(unsigned long long));
    spdp_status st = handle_alloc(h->device, at, &h->arrays);
    if (st != SPDP_OK) return st;
    char* base = static_cast<char*>(h->arrays.p);
    h->bitmap = reinterpret_cast<uint64_t*>(base + bitmap);
    h->colinfo = reinterpret_cast<uint32_t*>(base + colinfo);
    h->tileoffset = reinterpret_cast<uint32_t*>(base + tileoffset);
    if (h->q4) h->scales = reinterpret_cast<__half*>(base + scales);
    h->x_stage = reinterpret_cast<__half*>(base + x);
    h->mask_stage = reinterpret_cast<uint32_t*>(base + mask);
    h->y_stage = base + y;
    h->status_word = reinterpret_cast<int*>(base + status);
    h->pack_totals = reinterpret_cast<unsigned long long*>(h->status_word + 2);
    SPDP_CUDA_TRY(cudaMemsetAsync(h->status_word, 0, 2 * sizeof(int) + kPackTotals * sizeof(unsigned long long), s));
    return SPDP_OK;
}

// Chooses the number of CTAs (the kernel cuts the NGT GTiles into that many contiguous ranges) and (re)allocates what
// depends on it: the split-K workspaces (all zero = every tree node empty).  The caller synchronises `s`, so that the
// first call on any stream finds every tree node empty.
spdp_status build_partition(spdp_matrix* h, int num_ctas, cudaStream_t s) {
    const int64_t NGT = h->NGT;
    int P = num_ctas > 0 ? num_ctas : hostdev::default_ctas(h->R, h->C, h->sm_count * default_ctas_per_sm());
    if (P > 1024) P = 1024;          // the kernel's range arithmetic is 32-bit: NGT < 2^22 times P must fit
    if (P > NGT) P = static_cast<int>(NGT);
    if (P < 1) P = 1;
    const int64_t one = static_cast<int64_t>(P) * kTileM * sizeof(float);    // one row of split-K tree nodes per CTA
    const int64_t bytes = one + batch_workspace_bytes(P);
    // the new workspace first: where there is no memory for it the handle keeps the one it has
    DeviceBlock fresh = {};
    const spdp_status st = handle_alloc(h->device, bytes, &fresh);
    if (st != SPDP_OK) return st;
    const cudaError_t e = cudaMemsetAsync(fresh.p, 0, bytes, s);
    if (e != cudaSuccess) {
        handle_give(h->device, fresh, true);
        SPDP_CUDA_TRY(e);
    }
    handle_give(h->device, h->workspace_block, true);      // idle: a new handle has none, spdp_set_num_ctas has waited for the device
    h->workspace_block = fresh;
    h->workspace = static_cast<float*>(fresh.p);
    h->workspace_batch = h->workspace + P * kTileM;
    h->workspace_bytes = bytes;
    h->num_ctas = P;
    // a recorded host-vector call holds the old workspace and CTA count: it is recorded anew
    drop_host_graph(h);
    h->host_calls = 0;
    return SPDP_OK;
}

// The rest of a handle's set-up; synchronises `s`.
spdp_status finish_handle(spdp_matrix* h, cudaStream_t s) {
    spdp_status st = configure_spmspv_kernel();
    if (st != SPDP_OK) return st;
    st = configure_spmspv_batch_kernel();
    if (st != SPDP_OK) return st;
    st = configure_spmm_kernel();
    if (st != SPDP_OK) return st;
    st = configure_spmspv_q4_kernel();
    if (st != SPDP_OK) return st;
    SPDP_CUDA_TRY(cudaStreamSynchronize(s));
    handle_give(h->device, h->packing, true);
    return SPDP_OK;
}

bool misaligned(const void* p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

constexpr int64_t kMostSide = int64_t(1) << 30, kMostTokens = int64_t(1) << 24;
// Elements between rows of at least `row` (below 2^38, so that offsets of all tokens or weights fit 63 bits).
bool stride_ok(int64_t ld, int64_t row) { return ld >= row && ld <= (int64_t(1) << 38); }

// `count` weights of `rows` rows of `row` elements, none over another: one after another, row between row, or (0 apart) one for all.  Their last
// element is within 2^60 of the first.
bool weights_ok(int64_t count, int64_t apart, int64_t rows, int64_t ld, int64_t row) {
    constexpr int64_t kMostReach = int64_t(1) << 60;
    if (!stride_ok(ld, row) || rows - 1 > kMostReach / ld) return false;
    if (count == 1 || apart == 0) return true;
    if (!stride_ok(apart, row) || count - 1 > kMostReach / apart) return false;
    return (rows - 1) * ld + row <= apart || (count - 1) * apart + row <= ld;
}

constexpr int kMostCacheHeads = 4096, kMostRequests = 4096;
constexpr int64_t kMostPages = int64_t(1) << 28;
constexpr int64_t kMostKeys = INT32_MAX - 8192;         // of a request: the kernels look some thousands ahead of its last one
// A cache of 4-bit keys and values that the kernels take.
bool kv4_shape_ok(int kv_heads, int head_dim, int page_tokens) {
    return kv_heads >= 1 && kv_heads <= kMostCacheHeads && (head_dim == 64 || head_dim == 128 || head_dim == 256) && page_tokens >= 16 && page_tokens <= 256 &&
           (page_tokens & (page_tokens - 1)) == 0;
}

// The arguments that the calls on pages share.
spdp_status pages_call(KvPagesCall* c, void* ref, int64_t pages, void* table, int64_t rows, int64_t table_stride, int64_t table_pages, const void* a, const void* b, const void* d,
                       int64_t n, void* number_out) {
    if (ref == nullptr || table == nullptr || (n > 0 && (a == nullptr || b == nullptr || d == nullptr))) return SPDP_ERR_INVALID_ARG;
    if (pages < 1 || rows < 1 || table_pages < 1 || n < 0 || n > kMostRequests || !stride_ok(table_stride, table_pages)) return SPDP_ERR_INVALID_ARG;
    if (misaligned(ref, 3u) || misaligned(table, 3u) || misaligned(a, 3u) || misaligned(b, 3u) || misaligned(d, 3u) || misaligned(number_out, 3u)) return SPDP_ERR_INVALID_ARG;
    if (pages > kMostPages || rows > kMostTokens || table_pages > INT32_MAX / rows) return SPDP_ERR_UNSUPPORTED_SHAPE;
    c->ref = static_cast<int32_t*>(ref), c->table = static_cast<int32_t*>(table), c->short_out = static_cast<int32_t*>(number_out);
    c->row = static_cast<const int32_t*>(a), c->from = static_cast<const int32_t*>(b), c->to = static_cast<const int32_t*>(d);
    c->pages = pages, c->rows = rows, c->table_stride = table_stride, c->table_pages = table_pages, c->n = n;
    return SPDP_OK;
}
spdp_status pages_cache(KvPagesCall* c, void* cache, int layers, int64_t layer_stride, int64_t page_bytes, int64_t pages) {
    if (cache == nullptr || misaligned(cache, 15u) || layers < 1 || page_bytes < 16 || page_bytes % 16 != 0 || pages < 1) return SPDP_ERR_INVALID_ARG;
    if (pages > kMostPages || layers > 65536 || page_bytes > int64_t(1) << 32) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (layers > 1 && (layer_stride < pages * page_bytes || layer_stride % 16 != 0 || layer_stride > (int64_t(1) << 62) / layers)) return SPDP_ERR_INVALID_ARG;
    c->cache = static_cast<unsigned char*>(cache), c->layers = layers, c->layer_stride = layers > 1 ? layer_stride : 0, c->page_bytes = page_bytes, c->pages = pages;
    return SPDP_OK;
}

constexpr int kBatchViaSingleCalls = 2;   // spdp_spmspv_batch: up to this many tokens go through the single-vector kernel

// The decode kernel of the handle's Values variant (fp16 values, or 4-bit codes with scales).
spdp_status launch_decode(const spdp_matrix* h, const __half* x, int rule, float thr, const uint32_t* mask, void* y,
                          int ydt, cudaStream_t s) {
    return h->q4 ? launch_spmspv_q4(h, x, rule, thr, mask, y, ydt, s) : launch_spmspv(h, x, rule, thr, mask, y, ydt, s);
}

bool rule_ok(int rule) { return rule == SPDP_DP_NONE || rule == SPDP_DP_ABS_GT || rule == SPDP_DP_MASK; }

// copy in -> kernel -> copy out, enqueued on s.
spdp_status enqueue_host_call(spdp_matrix* h, const void* x_host, int rule, float thr, const void* mask_host,
                              void* y_host, int ydt, cudaStream_t s) {
    SPDP_CUDA_TRY(cudaMemcpyAsync(h->x_stage, x_host, h->K * sizeof(__half), cudaMemcpyHostToDevice, s));
    if (rule == SPDP_DP_MASK)
        SPDP_CUDA_TRY(cudaMemcpyAsync(h->mask_stage, mask_host, ((h->K + 31) / 32) * sizeof(uint32_t),
                                      cudaMemcpyHostToDevice, s));
    spdp_status st = launch_decode(h, h->x_stage, rule, thr, rule == SPDP_DP_MASK ? h->mask_stage : nullptr,
                                   h->y_stage, ydt, s);
    if (st != SPDP_OK) return st;
    const size_t ybytes = static_cast<size_t>(h->M) * (ydt == SPDP_Y_F32 ? sizeof(float) : sizeof(__half));
    SPDP_CUDA_TRY(cudaMemcpyAsync(y_host, h->y_stage, ybytes, cudaMemcpyDeviceToHost, s));
    return SPDP_OK;
}

// The page-locked range that holds a host address, asked of the driver in one call (looked up through the runtime: the library
// does not link libcuda).
using PointerAttributesFn = CUresult (*)(unsigned, CUpointer_attribute*, void**, CUdeviceptr);
PointerAttributesFn pointer_attributes_fn() {
    static PointerAttributesFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuPointerGetAttributes", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<PointerAttributesFn>(f);
    }();
    return fn;
}
hostdev::PinnedRange pinned_range(const void* p) {
    const PointerAttributesFn get = pointer_attributes_fn();
    unsigned type = 0, managed = 0;
    CUdeviceptr device = 0, start = 0;
    size_t size = 0;
    CUpointer_attribute what[] = {CU_POINTER_ATTRIBUTE_MEMORY_TYPE, CU_POINTER_ATTRIBUTE_IS_MANAGED, CU_POINTER_ATTRIBUTE_DEVICE_POINTER,
                                  CU_POINTER_ATTRIBUTE_RANGE_START_ADDR, CU_POINTER_ATTRIBUTE_RANGE_SIZE};
    void* out[] = {&type, &managed, &device, &start, &size};
    // pageable memory is no error here: every attribute comes back zero
    if (get == nullptr || get(5, what, out, reinterpret_cast<CUdeviceptr>(p)) != CUDA_SUCCESS || type != CU_MEMORYTYPE_HOST || managed != 0 || device == 0)
        return {0, 0, 0};
    return {static_cast<uint64_t>(start), static_cast<uint64_t>(size), static_cast<uint64_t>(device)};
}
// The address through which the kernels may use a host buffer, or null (see hostdev::direct_address).
void* direct_address(const void* p, size_t bytes, size_t align) {
    return reinterpret_cast<void*>(static_cast<uintptr_t>(hostdev::direct_address(reinterpret_cast<uintptr_t>(p), bytes, align, pinned_range(p))));
}

// The host-vector call with pinned buffers, whose device addresses the kernels use: a small kernel fetches x (and the mask) once, the
// decode kernel stores y over the bus.  No copy engine between the steps, and programmatic launch between the two kernels.
// us per call, copy engine -> this: 1024x1024 31 -> 20, 11008x4096 31 -> 27, 28672x8192 68 -> 62.  (Letting every CTA of the
// decode kernel read its part of x over the bus: 48 and 140 us on the last two, because every row tile reads x again.)
int mask_words(const spdp_matrix* h, int rule) { return rule == SPDP_DP_MASK ? static_cast<int>((h->K + 31) / 32) : 0; }
spdp_status enqueue_pinned_call(spdp_matrix* h, const spdp_matrix::HostCall& c, cudaStream_t s) {
    const int words = mask_words(h, c.rule);
    spdp_status st = launch_fetch(c.x, h->K, h->x_stage, c.mask, words, h->mask_stage, s);
    if (st != SPDP_OK) return st;
    return launch_decode(h, h->x_stage, c.rule, c.thr, words ? h->mask_stage : nullptr, c.y, c.ydt, s);
}

// Records the two kernels once (on a private stream) and keeps the instantiated graph: one launch instead of two saves
// 4 to 6 us of a call.
spdp_status record_host_graph(spdp_matrix* h, const spdp_matrix::HostCall& c) {
    if (h->capture_stream == nullptr)
        SPDP_CUDA_TRY(cudaStreamCreateWithFlags(&h->capture_stream, cudaStreamNonBlocking));
    SPDP_CUDA_TRY(cudaStreamBeginCapture(h->capture_stream, cudaStreamCaptureModeThreadLocal));
    spdp_status st = enqueue_pinned_call(h, c, h->capture_stream);
    cudaError_t e = cudaStreamEndCapture(h->capture_stream, &h->host_graph);
    size_t roots = 1, nodes = 2;
    cudaGraphNode_t all[2] = {};
    if (st == SPDP_OK && e == cudaSuccess) e = cudaGraphGetRootNodes(h->host_graph, &h->host_nodes[0], &roots);
    if (st == SPDP_OK && e == cudaSuccess) e = cudaGraphGetNodes(h->host_graph, all, &nodes);
    if (st == SPDP_OK && e == cudaSuccess) e = (roots == 1 && nodes == 2) ? cudaGraphInstantiate(&h->host_exec, h->host_graph, 0) : cudaErrorUnknown;
    if (st != SPDP_OK || e != cudaSuccess) {
        if (e != cudaSuccess) note_cuda_error(e, "recording the host-vector call");
        h->host_exec = nullptr;
        drop_host_graph(h);
        return st != SPDP_OK ? st : SPDP_ERR_CUDA;
    }
    h->host_nodes[1] = all[0] == h->host_nodes[0] ? all[1] : all[0];
    h->host_args = c;
    return SPDP_OK;
}

// Launches the recorded graph with the arguments of this call.
spdp_status replay_pinned_call(spdp_matrix* h, const spdp_matrix::HostCall& c, cudaStream_t s) {
    const int words = mask_words(h, c.rule);
    const spdp_matrix::HostCall& had = h->host_args;
    if (c.x != had.x || c.mask != had.mask || c.rule != had.rule) {
        const spdp_status st = set_fetch_node(h->host_exec, h->host_nodes[0], c.x, h->K, h->x_stage, c.mask, words, h->mask_stage);
        if (st != SPDP_OK) { drop_host_graph(h); return st; }
    }
    if (c.y != had.y || c.rule != had.rule || c.ydt != had.ydt || std::memcmp(&c.thr, &had.thr, sizeof(float)) != 0) {
        const auto set = h->q4 ? set_spmspv_q4_node : set_spmspv_node;
        const spdp_status st = set(h, h->host_exec, h->host_nodes[1], h->x_stage, c.rule, c.thr, words ? h->mask_stage : nullptr, c.y, c.ydt);
        if (st != SPDP_OK) { drop_host_graph(h); return st; }
    }
    h->host_args = c;
    SPDP_CUDA_TRY(cudaGraphLaunch(h->host_exec, s));
    return SPDP_OK;
}

}  // namespace
}  // namespace spdp

using namespace spdp;

extern "C" {

spdp_status spdp_pack_tiled_cbc_ex(const void* W_dev, int64_t M, int64_t K, int64_t ldw, int tile_m,
                                   int tile_k, int pad_elems, void* stream, spdp_handle* out) {
    if (W_dev == nullptr || out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (tile_m != kTileM || tile_k != kTileK) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (M < 1 || K < 1 || ldw < K) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (pad_elems != 8 && pad_elems != 1) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (reinterpret_cast<uintptr_t>(W_dev) & 1u) return SPDP_ERR_INVALID_ARG;
    spdp_matrix* h = nullptr;
    spdp_status st = new_handle(M, K, pad_elems, &h);
    if (st != SPDP_OK) return st;
    st = alloc_arrays(h, static_cast<cudaStream_t>(stream));
    if (st == SPDP_OK) st = build_partition(h, 0, static_cast<cudaStream_t>(stream));    // emptied before the kernels, not behind them
    if (st == SPDP_OK) st = pack_device(h, static_cast<const __half*>(W_dev), ldw, static_cast<cudaStream_t>(stream));
    if (st == SPDP_OK) st = finish_handle(h, static_cast<cudaStream_t>(stream));
    if (st != SPDP_OK) { release(h); return st; }
    *out = h;
    return SPDP_OK;
}

spdp_status spdp_pack_tiled_cbc(const void* W_dev, int64_t M, int64_t K, int64_t ldw, int tile_m,
                                int tile_k, void* stream, spdp_handle* out) {
    return spdp_pack_tiled_cbc_ex(W_dev, M, K, ldw, tile_m, tile_k, 8, stream, out);
}

spdp_status spdp_pack_tiled_cbc_q4(const void* W_dev, int64_t M, int64_t K, int64_t ldw, int tile_m, int tile_k,
                                   void* stream, spdp_handle* out) {
    if (W_dev == nullptr || out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (tile_m != kTileM || tile_k != kTileK) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (M < 1 || K < 1 || ldw < K) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (reinterpret_cast<uintptr_t>(W_dev) & 1u) return SPDP_ERR_INVALID_ARG;
    spdp_matrix* h = nullptr;
    spdp_status st = new_handle(M, K, 32, &h);
    if (st != SPDP_OK) return st;
    h->q4 = 1;
    st = alloc_arrays(h, static_cast<cudaStream_t>(stream));
    if (st == SPDP_OK) st = build_partition(h, 0, static_cast<cudaStream_t>(stream));    // emptied before the kernels, not behind them
    if (st == SPDP_OK) st = pack_device(h, static_cast<const __half*>(W_dev), ldw, static_cast<cudaStream_t>(stream));
    if (st == SPDP_OK) st = finish_handle(h, static_cast<cudaStream_t>(stream));
    if (st != SPDP_OK) { release(h); return st; }
    *out = h;
    return SPDP_OK;
}

spdp_status spdp_export_q4(spdp_handle h, void* tileoffset_host, void* colinfo_host, void* bitmap_host, void* codes_host,
                           void* scales_host) {
    if (!valid(h) || !h->q4) return SPDP_ERR_INVALID_ARG;
    SPDP_CUDA_TRY(cudaDeviceSynchronize());
    if (tileoffset_host)
        SPDP_CUDA_TRY(cudaMemcpy(tileoffset_host, h->tileoffset, (h->NGT + 1) * sizeof(uint32_t), cudaMemcpyDeviceToHost));
    if (colinfo_host)
        SPDP_CUDA_TRY(cudaMemcpy(colinfo_host, h->colinfo, h->NGT * kTileK * sizeof(uint32_t), cudaMemcpyDeviceToHost));
    if (bitmap_host)
        SPDP_CUDA_TRY(cudaMemcpy(bitmap_host, h->bitmap, h->NGT * kTileK * kWordsPerCol * sizeof(uint64_t),
                                 cudaMemcpyDeviceToHost));
    if (codes_host && h->values_len > 0)
        SPDP_CUDA_TRY(cudaMemcpy(codes_host, h->values, h->values_len / 2, cudaMemcpyDeviceToHost));
    if (scales_host)
        SPDP_CUDA_TRY(cudaMemcpy(scales_host, h->scales, h->NGT * kTileK * sizeof(__half), cudaMemcpyDeviceToHost));
    return SPDP_OK;
}

spdp_status spdp_import_tiled_cbc(int64_t M, int64_t K, int pad_elems, const void* tileoffset_host,
                                  const void* colinfo_host, const void* bitmap_host,
                                  const void* values_host, int64_t values_len, spdp_handle* out) {
    if (tileoffset_host == nullptr || colinfo_host == nullptr || bitmap_host == nullptr || out == nullptr)
        return SPDP_ERR_INVALID_ARG;
    if (values_len < 0 || (values_len > 0 && values_host == nullptr)) return SPDP_ERR_INVALID_ARG;
    if (values_len >= (int64_t(1) << 32)) return SPDP_ERR_OVERFLOW;
    spdp_matrix* h = nullptr;
    spdp_status st = new_handle(M, K, pad_elems, &h);
    if (st != SPDP_OK) return st;
    const uint32_t* to = static_cast<const uint32_t*>(tileoffset_host);
    const uint32_t* ci = static_cast<const uint32_t*>(colinfo_host);
    const uint64_t* bm = static_cast<const uint64_t*>(bitmap_host);
    // Structural validation of the arrays (Sec. 4.1): offsets are prefix sums of the padded counts.
    int64_t nnz = 0, uneven = 0;
    bool ok = (to[0] == 0) && (static_cast<int64_t>(to[h->NGT]) == values_len);
    for (int64_t g = 0; ok && g < h->NGT; ++g) {
        int64_t off = 0;
        for (int cc = 0; cc < kTileK; ++cc) {
            const int64_t slot = g * kTileK + cc;
            const int64_t n = ci[slot] & 0xFFFFu;
            int64_t pc = 0;
            for (int w = 0; w < kWordsPerCol; ++w) pc += __builtin_popcountll(bm[slot * kWordsPerCol + w]);
            if (static_cast<int64_t>(ci[slot] >> 16) != off || pc != n) { ok = false; break; }
            off += (n + pad_elems - 1) / pad_elems * pad_elems;
            nnz += n;
            const int64_t column = g % h->C * kTileK + cc, diff = n - static_cast<int64_t>(ci[slot ^ 1] & 0xFFFFu);
            if ((column | 1) < K) uneven += diff * diff;
        }
        if (ok && static_cast<int64_t>(to[g + 1]) - static_cast<int64_t>(to[g]) != off) ok = false;
    }
    if (!ok) { release(h); return SPDP_ERR_INVALID_ARG; }
    h->nnz = nnz;
    h->uneven = uneven;
    h->values_len = values_len;
    const size_t vbytes = static_cast<size_t>(values_len) * sizeof(__half);
    auto body = [&]() -> spdp_status {
        cudaStream_t s = nullptr;
        spdp_status a = alloc_arrays(h, s);
        if (a == SPDP_OK) a = build_partition(h, 0, s);
        if (a == SPDP_OK) a = handle_alloc(h->device, vbytes < 16 ? 16 : vbytes, &h->values_block);
        if (a != SPDP_OK) return a;
        h->values = static_cast<__half*>(h->values_block.p);
        SPDP_CUDA_TRY(cudaStreamSynchronize(s));
        SPDP_CUDA_TRY(cudaMemcpy(h->tileoffset, to, (h->NGT + 1) * sizeof(uint32_t), cudaMemcpyHostToDevice));
        SPDP_CUDA_TRY(cudaMemcpy(h->colinfo, ci, h->NGT * kTileK * sizeof(uint32_t), cudaMemcpyHostToDevice));
        SPDP_CUDA_TRY(cudaMemcpy(h->bitmap, bm, h->NGT * kTileK * kWordsPerCol * sizeof(uint64_t),
                                 cudaMemcpyHostToDevice));
        if (vbytes) SPDP_CUDA_TRY(cudaMemcpy(h->values, values_host, vbytes, cudaMemcpyHostToDevice));
        return finish_handle(h, s);
    };
    st = body();
    if (st != SPDP_OK) { release(h); return st; }
    *out = h;
    return SPDP_OK;
}

spdp_status spdp_spmspv(spdp_handle h, const void* x_dev, spdp_dp_rule rule, float thr,
                        const void* mask_dev, void* y_dev, spdp_ydtype ydt, void* stream) {
    if (!valid(h) || x_dev == nullptr || y_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!rule_ok(rule) || (ydt != SPDP_Y_F16 && ydt != SPDP_Y_F32)) return SPDP_ERR_INVALID_ARG;
    if (rule == SPDP_DP_MASK && mask_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(x_dev) & 1u) ||
        (reinterpret_cast<uintptr_t>(y_dev) & (ydt == SPDP_Y_F32 ? 3u : 1u)) ||
        (reinterpret_cast<uintptr_t>(mask_dev) & 3u))
        return SPDP_ERR_INVALID_ARG;
    if (h->pad_elems != 8 && !h->q4) return SPDP_ERR_UNSUPPORTED_SHAPE;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != h->device) return SPDP_ERR_INVALID_ARG;   // wrong current device
    return launch_decode(h, static_cast<const __half*>(x_dev), rule, thr,
                         static_cast<const uint32_t*>(mask_dev), y_dev, ydt, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_spmspv_batch(spdp_handle h, const void* x_dev, int64_t ldx, int batch, spdp_dp_rule rule, float thr,
                              const void* mask_dev, int64_t mask_stride, void* y_dev, int64_t ldy,
                              spdp_ydtype ydt, void* stream) {
    if (!valid(h) || x_dev == nullptr || y_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (batch < 1 || batch > SPDP_MAX_BATCH || ldx < h->K || ldy < h->M) return SPDP_ERR_INVALID_ARG;
    if (!rule_ok(rule) || (ydt != SPDP_Y_F16 && ydt != SPDP_Y_F32)) return SPDP_ERR_INVALID_ARG;
    if (rule == SPDP_DP_MASK && (mask_dev == nullptr || mask_stride < (h->K + 31) / 32)) return SPDP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(x_dev) & 1u) ||
        (reinterpret_cast<uintptr_t>(y_dev) & (ydt == SPDP_Y_F32 ? 3u : 1u)) ||
        (reinterpret_cast<uintptr_t>(mask_dev) & 3u))
        return SPDP_ERR_INVALID_ARG;
    if (h->pad_elems != 8) return SPDP_ERR_UNSUPPORTED_SHAPE;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != h->device) return SPDP_ERR_INVALID_ARG;   // wrong current device
    const __half* x = static_cast<const __half*>(x_dev);
    const uint32_t* mask = static_cast<const uint32_t*>(mask_dev);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (batch <= kBatchViaSingleCalls) {
        // The batch kernel's cost per fetched column tile does not depend on the number of tokens; below
        // three tokens one single-vector launch per token is faster (measured: 91 against 102 us for two
        // tokens on the 28672 x 8192 layer).  Same stream, same handle: the launches run in order.
        const size_t ybytes = ydt == SPDP_Y_F32 ? sizeof(float) : sizeof(__half);
        for (int b = 0; b < batch; ++b) {
            spdp_status st = launch_spmspv(h, x + b * ldx, rule, thr, mask ? mask + b * mask_stride : nullptr,
                                           static_cast<unsigned char*>(y_dev) + b * ldy * ybytes, ydt, s);
            if (st != SPDP_OK) return st;
        }
        return SPDP_OK;
    }
    return launch_spmspv_batch(h, x, ldx, batch, rule, thr, mask, mask_stride, y_dev, ldy, ydt, s);
}

spdp_status spdp_spmm(spdp_handle h, const void* X_dev, int64_t N, int64_t ldx, void* Y_dev, int64_t ldy,
                      spdp_ydtype ydt, void* stream) {
    if (!valid(h) || X_dev == nullptr || Y_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (N < 1 || N > (int64_t(1) << 24) || ldx < h->K || ldy < h->M) return SPDP_ERR_INVALID_ARG;
    if (ydt != SPDP_Y_F16 && ydt != SPDP_Y_F32) return SPDP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(X_dev) & 15u) || (ldx & 7) ||
        (reinterpret_cast<uintptr_t>(Y_dev) & (ydt == SPDP_Y_F32 ? 3u : 1u)))
        return SPDP_ERR_INVALID_ARG;
    if (h->pad_elems != 8) return SPDP_ERR_UNSUPPORTED_SHAPE;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != h->device) return SPDP_ERR_INVALID_ARG;   // wrong current device
    return launch_spmm(h, static_cast<const __half*>(X_dev), N, ldx, Y_dev, ldy, ydt, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_spmspv_noalloc(const void* tileoffset_dev, const void* colinfo_dev, const void* bitmap_dev,
                                const void* values_dev, int64_t M, int64_t K, const void* x_dev,
                                spdp_dp_rule rule, float thr, const void* mask_dev, void* y_dev,
                                spdp_ydtype ydt, void* stream) {
    if (tileoffset_dev == nullptr || colinfo_dev == nullptr || bitmap_dev == nullptr || values_dev == nullptr ||
        x_dev == nullptr || y_dev == nullptr)
        return SPDP_ERR_INVALID_ARG;
    if (M < 1 || K < 1) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (!rule_ok(rule) || (ydt != SPDP_Y_F16 && ydt != SPDP_Y_F32)) return SPDP_ERR_INVALID_ARG;
    if (rule == SPDP_DP_MASK && mask_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(values_dev) & 15u) || (reinterpret_cast<uintptr_t>(bitmap_dev) & 7u) ||
        (reinterpret_cast<uintptr_t>(tileoffset_dev) & 3u) || (reinterpret_cast<uintptr_t>(colinfo_dev) & 15u) ||
        (reinterpret_cast<uintptr_t>(x_dev) & 1u) || (reinterpret_cast<uintptr_t>(mask_dev) & 3u) ||
        (reinterpret_cast<uintptr_t>(y_dev) & (ydt == SPDP_Y_F32 ? 3u : 1u)))
        return SPDP_ERR_INVALID_ARG;
    return launch_spmspv_noalloc(static_cast<const uint32_t*>(tileoffset_dev), static_cast<const uint32_t*>(colinfo_dev),
                                 static_cast<const uint64_t*>(bitmap_dev), static_cast<const __half*>(values_dev), M, K,
                                 static_cast<const __half*>(x_dev), rule, thr, static_cast<const uint32_t*>(mask_dev),
                                 y_dev, ydt, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_spmspv_host(spdp_handle h, const void* x_host, spdp_dp_rule rule, float thr,
                             const void* mask_host, void* y_host, spdp_ydtype ydt, void* stream) {
    if (!valid(h) || x_host == nullptr || y_host == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!rule_ok(rule) || (ydt != SPDP_Y_F16 && ydt != SPDP_Y_F32)) return SPDP_ERR_INVALID_ARG;
    if (rule == SPDP_DP_MASK && mask_host == nullptr) return SPDP_ERR_INVALID_ARG;
    if (h->pad_elems != 8 && !h->q4) return SPDP_ERR_UNSUPPORTED_SHAPE;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != h->device) return SPDP_ERR_INVALID_ARG;   // wrong current device
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // What is pinned is looked up on every call, and every call's arguments go into the recorded graph: nothing is assumed
    // about a buffer because an earlier one had its address.  A buffer that a kernel may not touch takes the copies.
    spdp_matrix::HostCall c = {};
    c.rule = rule;
    c.thr = thr;
    c.ydt = ydt;
    const size_t ysize = ydt == SPDP_Y_F32 ? sizeof(float) : sizeof(__half);
    c.x = static_cast<const __half*>(direct_address(x_host, h->K * sizeof(__half), sizeof(__half)));
    c.y = c.x != nullptr ? direct_address(y_host, h->M * ysize, ysize) : nullptr;
    if (rule == SPDP_DP_MASK && c.y != nullptr)
        c.mask = static_cast<const uint32_t*>(direct_address(mask_host, mask_words(h, rule) * sizeof(uint32_t), sizeof(uint32_t)));
    spdp_status st;
    if (c.y == nullptr || (rule == SPDP_DP_MASK && c.mask == nullptr)) {
        st = enqueue_host_call(h, x_host, rule, thr, mask_host, y_host, ydt, s);
    } else {
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        const bool capturing = cudaStreamIsCapturing(s, &cap) != cudaSuccess || cap != cudaStreamCaptureStatusNone;
        // a handle that is called again gets its graph (recording takes longer than one call saves)
        if (!capturing && h->host_exec == nullptr && ++h->host_calls == 2 && record_host_graph(h, c) != SPDP_OK) cudaGetLastError();
        st = (!capturing && h->host_exec != nullptr) ? replay_pinned_call(h, c, s) : enqueue_pinned_call(h, c, s);
    }
    if (st != SPDP_OK) return st;
    SPDP_CUDA_TRY(cudaStreamSynchronize(s));
    return SPDP_OK;
}

spdp_status spdp_swiglu_dp(const void* gate_dev, const void* up_dev, int64_t K, float thr, void* x_dev_out,
                           void* mask_dev_out, void* count_dev_out, void* stream) {
    if (gate_dev == nullptr || up_dev == nullptr || x_dev_out == nullptr || mask_dev_out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (K < 1 || K > (int64_t(1) << 30)) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if ((reinterpret_cast<uintptr_t>(gate_dev) & 1u) || (reinterpret_cast<uintptr_t>(up_dev) & 1u) ||
        (reinterpret_cast<uintptr_t>(x_dev_out) & 1u) || (reinterpret_cast<uintptr_t>(mask_dev_out) & 3u) ||
        (reinterpret_cast<uintptr_t>(count_dev_out) & 3u))
        return SPDP_ERR_INVALID_ARG;
    return launch_swiglu_dp(static_cast<const __half*>(gate_dev), static_cast<const __half*>(up_dev), K, thr,
                            static_cast<__half*>(x_dev_out), static_cast<uint32_t*>(mask_dev_out),
                            static_cast<int*>(count_dev_out), static_cast<cudaStream_t>(stream));
}

spdp_status spdp_lora(const void* X_dev, int64_t N, int64_t K, int64_t ldx, const void* adapter_dev, const void* A_dev, int64_t lda,
                      int64_t stride_a, const void* B_dev, int64_t ldb, int64_t stride_b, int64_t count, int rank, const void* ranks_dev,
                      const void* scales_dev, const void* base_dev, int64_t ldbase, void* Y_dev, int64_t M, int64_t ldy, spdp_ydtype ydt,
                      void* stream) {
    if (X_dev == nullptr || adapter_dev == nullptr || A_dev == nullptr || B_dev == nullptr || base_dev == nullptr || Y_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (K < 1 || M < 1 || K > kMostSide || M > kMostSide || rank < 1 || rank > SPDP_MAX_RANK) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (N < 1 || N > kMostTokens || count < 1 || count > INT32_MAX) return SPDP_ERR_INVALID_ARG;
    if (!stride_ok(ldx, K) || !stride_ok(ldbase, M) || !stride_ok(ldy, M) || !weights_ok(count, stride_a, rank, lda, K) || !weights_ok(count, stride_b, M, ldb, rank))
        return SPDP_ERR_INVALID_ARG;
    if ((ydt != SPDP_Y_F16 && ydt != SPDP_Y_F32) || (base_dev == Y_dev && N > 1 && ldbase != ldy)) return SPDP_ERR_INVALID_ARG;
    const unsigned y = ydt == SPDP_Y_F32 ? 3u : 1u;
    if (misaligned(X_dev, 1u) || misaligned(A_dev, 1u) || misaligned(B_dev, 1u) || misaligned(base_dev, y) || misaligned(Y_dev, y) || misaligned(adapter_dev, 3u) ||
        misaligned(ranks_dev, 3u) || misaligned(scales_dev, 3u))
        return SPDP_ERR_INVALID_ARG;
    LoraCall c = {};
    c.X = static_cast<const __half*>(X_dev), c.adapter = static_cast<const int32_t*>(adapter_dev), c.A = static_cast<const __half*>(A_dev);
    c.B = static_cast<const __half*>(B_dev), c.ranks = static_cast<const int32_t*>(ranks_dev), c.scales = static_cast<const float*>(scales_dev);
    c.base = base_dev, c.Y = Y_dev, c.N = N, c.K = K, c.M = M, c.count = count, c.ldx = ldx, c.lda = lda, c.stride_a = count > 1 ? stride_a : 0, c.ldb = ldb;
    c.stride_b = count > 1 ? stride_b : 0, c.ldbase = ldbase, c.ldy = ldy, c.rank = rank, c.ydt = ydt;
    return launch_lora(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_qk_norm_rope(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, spdp_ydtype dt, int64_t N, int q_heads, int kv_heads,
                              int head_dim, const void* q_weight_dev, const void* k_weight_dev, float eps, const void* pos_dev, int64_t pos_stride,
                              int axes, const int* sections, const void* inv_freq_dev, int pairs, int adjacent, void* q_out_dev,
                              int64_t ldq_out, void* k_out_dev, int64_t ldk_out, void* stream) {
    constexpr int kMostHeads = 1 << 16, kMostAxes = 4;
    if (head_dim < 2 || head_dim > 256 || head_dim % 2 != 0 || q_heads > kMostHeads || kv_heads > kMostHeads) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (N < 1 || N > kMostTokens || q_heads < 0 || kv_heads < 0 || q_heads + kv_heads < 1) return SPDP_ERR_INVALID_ARG;
    if (dt != SPDP_Y_F16 && dt != SPDP_Y_F32) return SPDP_ERR_INVALID_ARG;
    if (pairs < 0 || pairs > head_dim / 2 || (adjacent != 0 && adjacent != 1) || !(eps >= 0.0f)) return SPDP_ERR_INVALID_ARG;
    const unsigned in = dt == SPDP_Y_F32 ? 3u : 1u;
    const int64_t q_row = static_cast<int64_t>(q_heads) * head_dim, k_row = static_cast<int64_t>(kv_heads) * head_dim;
    if (q_heads > 0 && (q_dev == nullptr || q_out_dev == nullptr || !stride_ok(ldq, q_row) || !stride_ok(ldq_out, q_row) || misaligned(q_dev, in) ||
                        misaligned(q_out_dev, 1u) || misaligned(q_weight_dev, 1u) || (q_out_dev == q_dev && (dt != SPDP_Y_F16 || (N > 1 && ldq != ldq_out)))))
        return SPDP_ERR_INVALID_ARG;
    if (kv_heads > 0 && (k_dev == nullptr || k_out_dev == nullptr || !stride_ok(ldk, k_row) || !stride_ok(ldk_out, k_row) || misaligned(k_dev, in) ||
                         misaligned(k_out_dev, 1u) || misaligned(k_weight_dev, 1u) || (k_out_dev == k_dev && (dt != SPDP_Y_F16 || (N > 1 && ldk != ldk_out)))))
        return SPDP_ERR_INVALID_ARG;
    if (pairs > 0) {
        if (pos_dev == nullptr || inv_freq_dev == nullptr || sections == nullptr || axes < 1 || axes > kMostAxes || !stride_ok(pos_stride, N) || misaligned(pos_dev, 3u) ||
            misaligned(inv_freq_dev, 3u))
            return SPDP_ERR_INVALID_ARG;
        int64_t sum = 0;
        for (int a = 0; a < axes; ++a) {
            if (sections[a] < 0) return SPDP_ERR_INVALID_ARG;
            sum += sections[a];
        }
        if (sum != pairs) return SPDP_ERR_INVALID_ARG;
    }
    HeadsCall c = {};
    if (q_heads > 0) c.q = q_dev, c.q_out = static_cast<__half*>(q_out_dev), c.q_weight = static_cast<const __half*>(q_weight_dev), c.ldq = ldq, c.ldq_out = ldq_out;
    if (kv_heads > 0) c.k = k_dev, c.k_out = static_cast<__half*>(k_out_dev), c.k_weight = static_cast<const __half*>(k_weight_dev), c.ldk = ldk, c.ldk_out = ldk_out;
    if (pairs > 0) {
        c.pos = static_cast<const int32_t*>(pos_dev), c.inv_freq = static_cast<const float*>(inv_freq_dev);
        c.sections = sections, c.pos_stride = pos_stride, c.axes = axes;
    }
    c.N = N, c.q_heads = q_heads, c.kv_heads = kv_heads, c.head_dim = head_dim, c.pairs = pairs, c.dt = dt, c.eps = eps, c.adjacent = adjacent != 0;
    return launch_qk_norm_rope(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv4_page_bytes(int kv_heads, int head_dim, int page_tokens, int64_t* bytes_out) {
    if (bytes_out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!kv4_shape_ok(kv_heads, head_dim, page_tokens)) return SPDP_ERR_UNSUPPORTED_SHAPE;
    *bytes_out = static_cast<int64_t>(kv_heads) * page_tokens * (head_dim + head_dim / 8);
    return SPDP_OK;
}

spdp_status spdp_kv4_store(const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv, spdp_ydtype vdt, int64_t N, int kv_heads, int head_dim,
                           const void* slot_dev, void* cache_dev, int64_t pages, int page_tokens, void* k_values_dev_out, int64_t ldk_values,
                           void* v_values_dev_out, int64_t ldv_values, void* stream) {
    if (k_dev == nullptr || v_dev == nullptr || slot_dev == nullptr || cache_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!kv4_shape_ok(kv_heads, head_dim, page_tokens)) return SPDP_ERR_UNSUPPORTED_SHAPE;
    const int64_t row = static_cast<int64_t>(kv_heads) * head_dim;
    if (N < 1 || N > kMostTokens || pages < 1 || pages > INT32_MAX || !stride_ok(ldk, row) || !stride_ok(ldv, row) || (vdt != SPDP_Y_F16 && vdt != SPDP_Y_F32))
        return SPDP_ERR_INVALID_ARG;
    if ((k_values_dev_out != nullptr && !stride_ok(ldk_values, row)) || (v_values_dev_out != nullptr && !stride_ok(ldv_values, row))) return SPDP_ERR_INVALID_ARG;
    if (misaligned(k_dev, 1u) || misaligned(v_dev, vdt == SPDP_Y_F32 ? 3u : 1u) || misaligned(slot_dev, 7u) || misaligned(cache_dev, 15u) ||
        misaligned(k_values_dev_out, 1u) || misaligned(v_values_dev_out, 1u))
        return SPDP_ERR_INVALID_ARG;
    Kv4StoreCall c = {};
    c.k = static_cast<const __half*>(k_dev), c.v = v_dev, c.slot = static_cast<const int64_t*>(slot_dev), c.cache = static_cast<unsigned char*>(cache_dev);
    c.k_values = static_cast<__half*>(k_values_dev_out), c.v_values = static_cast<__half*>(v_values_dev_out);
    c.N = N, c.ldk = ldk, c.ldv = ldv, c.pages = pages;
    c.ldk_values = k_values_dev_out != nullptr ? ldk_values : 0, c.ldv_values = v_values_dev_out != nullptr ? ldv_values : 0;
    c.kv_heads = kv_heads, c.head_dim = head_dim, c.page_tokens = page_tokens, c.vdt = vdt;
    return launch_kv4_store(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_attn_kv4(const void* q_dev, int64_t ldq, int64_t B, int q_heads, int kv_heads, int head_dim, const void* cache_dev, int64_t pages,
                          int page_tokens, const void* table_dev, int64_t table_stride, int64_t table_pages, const void* length_dev, float scale,
                          float cap, int64_t window, float thr, void* y_dev, int64_t ldy, void* mask_dev_out, int64_t mask_stride, void* stream) {
    if (q_dev == nullptr || cache_dev == nullptr || table_dev == nullptr || length_dev == nullptr || y_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!kv4_shape_ok(kv_heads, head_dim, page_tokens) || q_heads < 1 || q_heads > 16 * kMostCacheHeads || q_heads % kv_heads != 0) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (B < 1 || B > 4096) return SPDP_ERR_UNSUPPORTED_SHAPE;
    const int64_t row = static_cast<int64_t>(q_heads) * head_dim;
    if (pages < 1 || pages > INT32_MAX || table_pages < 1 || !stride_ok(table_stride, table_pages) || !stride_ok(ldq, row) || !stride_ok(ldy, row) || window < 0)
        return SPDP_ERR_INVALID_ARG;
    if (mask_dev_out != nullptr && !stride_ok(mask_stride, row / 32)) return SPDP_ERR_INVALID_ARG;
    // products are below 2^41, so scores stay below the 10^30 that stands for "no score yet" in the kernel
    if (!(scale >= -1.0e16f && scale <= 1.0e16f) || !(cap >= 0.0f && cap <= 1.0e38f)) return SPDP_ERR_INVALID_ARG;
    if (misaligned(q_dev, 1u) || misaligned(cache_dev, 15u) || misaligned(table_dev, 3u) || misaligned(length_dev, 3u) || misaligned(y_dev, 1u) ||
        misaligned(mask_dev_out, 3u))
        return SPDP_ERR_INVALID_ARG;
    // the keys of a request (the kernel looks up to 4200 of them ahead of its last one), and the 64-key units of all requests and heads
    // with what the kernel adds to each (7 at most, a part of a unit among them), are counted in 32 bits
    if (table_pages > (INT32_MAX - 8192) / page_tokens) return SPDP_ERR_UNSUPPORTED_SHAPE;
    const int64_t triples = kv_heads * static_cast<int64_t>((q_heads / kv_heads + 7) / 8);
    if (triples * (table_pages * page_tokens / 64 + 8) > INT32_MAX / B) return SPDP_ERR_UNSUPPORTED_SHAPE;
    Kv4AttnCall c = {};
    c.q = static_cast<const __half*>(q_dev), c.cache = static_cast<const unsigned char*>(cache_dev), c.table = static_cast<const int32_t*>(table_dev);
    c.length = static_cast<const int32_t*>(length_dev), c.y = static_cast<__half*>(y_dev), c.mask = static_cast<uint32_t*>(mask_dev_out);
    c.B = B, c.ldq = ldq, c.ldy = ldy, c.table_stride = table_stride, c.table_pages = table_pages, c.mask_stride = mask_stride, c.pages = pages, c.window = window;
    c.q_heads = q_heads, c.kv_heads = kv_heads, c.head_dim = head_dim, c.page_tokens = page_tokens, c.scale = scale, c.cap = cap, c.thr = thr;
    return launch_attn_kv4(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv8_page_bytes(int kv_heads, int head_dim, int page_tokens, int64_t* bytes_out) {
    if (bytes_out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!kv4_shape_ok(kv_heads, head_dim, page_tokens)) return SPDP_ERR_UNSUPPORTED_SHAPE;
    *bytes_out = static_cast<int64_t>(kv_heads) * page_tokens * (2 * head_dim + 1);
    return SPDP_OK;
}

spdp_status spdp_kv8_store(const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv, spdp_ydtype vdt, int64_t N, int kv_heads, int head_dim, int64_t B,
                           const void* first_dev, const void* table_dev, int64_t table_stride, int64_t table_pages, const void* length_dev, void* cache_dev,
                           int64_t pages, int page_tokens, void* k_values_dev_out, int64_t ldk_values, void* v_values_dev_out, int64_t ldv_values, void* stream) {
    if (k_dev == nullptr || v_dev == nullptr || table_dev == nullptr || length_dev == nullptr || cache_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!kv4_shape_ok(kv_heads, head_dim, page_tokens) || B > kMostRequests) return SPDP_ERR_UNSUPPORTED_SHAPE;
    const int64_t row = static_cast<int64_t>(kv_heads) * head_dim;
    if (N < 1 || N > kMostTokens || B < 1 || (first_dev == nullptr && B != N) || pages < 1 || pages > INT32_MAX || table_pages < 1 || !stride_ok(table_stride, table_pages) ||
        !stride_ok(ldk, row) || !stride_ok(ldv, row) || (vdt != SPDP_Y_F16 && vdt != SPDP_Y_F32))
        return SPDP_ERR_INVALID_ARG;
    if ((k_values_dev_out != nullptr && !stride_ok(ldk_values, row)) || (v_values_dev_out != nullptr && !stride_ok(ldv_values, row))) return SPDP_ERR_INVALID_ARG;
    if (misaligned(k_dev, 1u) || misaligned(v_dev, vdt == SPDP_Y_F32 ? 3u : 1u) || misaligned(first_dev, 3u) || misaligned(table_dev, 3u) || misaligned(length_dev, 3u) ||
        misaligned(cache_dev, 15u) || misaligned(k_values_dev_out, 1u) || misaligned(v_values_dev_out, 1u))
        return SPDP_ERR_INVALID_ARG;
    if (table_pages > kMostKeys / page_tokens) return SPDP_ERR_UNSUPPORTED_SHAPE;
    Kv8StoreCall c = {};
    c.k = static_cast<const __half*>(k_dev), c.v = v_dev, c.first = static_cast<const int32_t*>(first_dev), c.table = static_cast<const int32_t*>(table_dev);
    c.length = static_cast<const int32_t*>(length_dev), c.cache = static_cast<unsigned char*>(cache_dev);
    c.k_values = static_cast<__half*>(k_values_dev_out), c.v_values = static_cast<__half*>(v_values_dev_out);
    c.N = N, c.B = B, c.ldk = ldk, c.ldv = ldv, c.pages = pages, c.table_stride = table_stride, c.table_pages = table_pages;
    c.ldk_values = k_values_dev_out != nullptr ? ldk_values : 0, c.ldv_values = v_values_dev_out != nullptr ? ldv_values : 0;
    c.kv_heads = kv_heads, c.head_dim = head_dim, c.page_tokens = page_tokens, c.vdt = vdt;
    return launch_kv8_store(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_attn_kv8(const void* q_dev, int64_t ldq, int64_t N, int q_heads, int kv_heads, int head_dim, int64_t B, const void* first_dev, const void* cache_dev,
                          int64_t pages, int page_tokens, const void* table_dev, int64_t table_stride, int64_t table_pages, const void* length_dev, float scale, float cap,
                          int64_t window, int64_t sinks, float thr, void* y_dev, int64_t ldy, void* mask_dev_out, int64_t mask_stride, void* stream) {
    if (q_dev == nullptr || cache_dev == nullptr || table_dev == nullptr || length_dev == nullptr || y_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!kv4_shape_ok(kv_heads, head_dim, page_tokens) || q_heads < 1 || q_heads > 16 * kMostCacheHeads || q_heads % kv_heads != 0) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (B > kMostRequests) return SPDP_ERR_UNSUPPORTED_SHAPE;
    const int64_t row = static_cast<int64_t>(q_heads) * head_dim;
    if (N < 1 || N > kMostTokens || B < 1 || (first_dev == nullptr && B != N) || pages < 1 || pages > INT32_MAX || table_pages < 1 || !stride_ok(table_stride, table_pages) ||
        !stride_ok(ldq, row) || !stride_ok(ldy, row) || window < 0 || sinks < 0)
        return SPDP_ERR_INVALID_ARG;
    if (mask_dev_out != nullptr && !stride_ok(mask_stride, row / 32)) return SPDP_ERR_INVALID_ARG;
    // products are below 2^41, so scores stay below the 10^30 that stands for "no score yet" in the kernel
    if (!(scale >= -1.0e16f && scale <= 1.0e16f) || !(cap >= 0.0f && cap <= 1.0e38f)) return SPDP_ERR_INVALID_ARG;
    if (misaligned(q_dev, 1u) || misaligned(first_dev, 3u) || misaligned(cache_dev, 15u) || misaligned(table_dev, 3u) || misaligned(length_dev, 3u) || misaligned(y_dev, 1u) ||
        misaligned(mask_dev_out, 3u))
        return SPDP_ERR_INVALID_ARG;
    // the keys of a request, the rows of all and the units of keys of all blocks of rows, with what the kernels add, are counted in 32 bits
    if (table_pages > kMostKeys / page_tokens || N > INT32_MAX / q_heads) return SPDP_ERR_UNSUPPORTED_SHAPE;
    const int64_t group = q_heads / kv_heads, keys = table_pages * page_tokens, few = first_dev == nullptr ? group : N * group < kFewRows ? N * group : kFewRows;
    if (kv_heads * ((few + 7) / 8) * (keys / 64 + 8) > INT32_MAX / B) return SPDP_ERR_UNSUPPORTED_SHAPE;
    if (first_dev != nullptr && kv_heads * (N * group / 128 + B) > INT32_MAX / (keys / 128 + 8)) return SPDP_ERR_UNSUPPORTED_SHAPE;
    Kv8AttnCall c = {};
    c.q = static_cast<const __half*>(q_dev), c.cache = static_cast<const unsigned char*>(cache_dev), c.first = static_cast<const int32_t*>(first_dev);
    c.table = static_cast<const int32_t*>(table_dev), c.length = static_cast<const int32_t*>(length_dev), c.y = static_cast<__half*>(y_dev), c.mask = static_cast<uint32_t*>(mask_dev_out);
    c.N = N, c.B = B, c.ldq = ldq, c.ldy = ldy, c.table_stride = table_stride, c.table_pages = table_pages, c.mask_stride = mask_stride, c.pages = pages;
    c.window = window, c.sinks = sinks, c.q_heads = q_heads, c.kv_heads = kv_heads, c.head_dim = head_dim, c.page_tokens = page_tokens;
    c.scale = scale, c.cap = cap, c.thr = thr;
    return launch_attn_kv8(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv_pages_take(void* ref_dev, int64_t pages, void* table_dev, int64_t rows, int64_t table_stride, int64_t table_pages, const void* row_dev,
                               const void* from_dev, const void* to_dev, int64_t n, void* short_dev_out, void* stream) {
    KvPagesCall c = {};
    const spdp_status st = pages_call(&c, ref_dev, pages, table_dev, rows, table_stride, table_pages, row_dev, from_dev, to_dev, n, short_dev_out);
    return st != SPDP_OK ? st : launch_kv_pages_take(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv_pages_free(void* ref_dev, int64_t pages, void* table_dev, int64_t rows, int64_t table_stride, int64_t table_pages, const void* row_dev,
                               const void* from_dev, const void* to_dev, int64_t n, void* stream) {
    KvPagesCall c = {};
    const spdp_status st = pages_call(&c, ref_dev, pages, table_dev, rows, table_stride, table_pages, row_dev, from_dev, to_dev, n, nullptr);
    return st != SPDP_OK ? st : launch_kv_pages_free(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv_pages_fork(void* cache_dev, int layers, int64_t layer_stride, int64_t page_bytes, void* ref_dev, int64_t pages, void* table_dev, int64_t rows,
                               int64_t table_stride, int64_t table_pages, int page_tokens, const void* parent_dev, const void* child_dev, const void* length_dev, int64_t n,
                               void* short_dev_out, void* stream) {
    KvPagesCall c = {};
    spdp_status st = pages_call(&c, ref_dev, pages, table_dev, rows, table_stride, table_pages, parent_dev, child_dev, length_dev, n, short_dev_out);
    if (st == SPDP_OK) st = pages_cache(&c, cache_dev, layers, layer_stride, page_bytes, pages);
    if (st != SPDP_OK) return st;
    if (page_tokens < 1 || page_tokens > 1 << 16 || (page_tokens & (page_tokens - 1)) != 0) return SPDP_ERR_UNSUPPORTED_SHAPE;
    c.page_tokens = page_tokens;
    return launch_kv_pages_fork(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv_pages_copy(void* cache_dev, int layers, int64_t layer_stride, int64_t page_bytes, int64_t pages, const void* src_dev, const void* dst_dev, int64_t n,
                               void* stream) {
    KvPagesCall c = {};
    const spdp_status st = pages_cache(&c, cache_dev, layers, layer_stride, page_bytes, pages);
    if (st != SPDP_OK) return st;
    if (n < 0 || n > kMostRequests || (n > 0 && (src_dev == nullptr || dst_dev == nullptr)) || misaligned(src_dev, 3u) || misaligned(dst_dev, 3u)) return SPDP_ERR_INVALID_ARG;
    c.row = static_cast<const int32_t*>(src_dev), c.to = static_cast<const int32_t*>(dst_dev), c.n = n;
    return launch_kv_pages_copy(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_kv_pages_compact(void* cache_dev, int layers, int64_t layer_stride, int64_t page_bytes, void* ref_dev, int64_t pages, void* table_dev, int64_t rows,
                                  int64_t table_stride, int64_t table_pages, void* live_dev_out, void* stream) {
    KvPagesCall c = {};
    spdp_status st = pages_call(&c, ref_dev, pages, table_dev, rows, table_stride, table_pages, nullptr, nullptr, nullptr, 0, live_dev_out);
    if (st == SPDP_OK) st = pages_cache(&c, cache_dev, layers, layer_stride, page_bytes, pages);
    return st != SPDP_OK ? st : launch_kv_pages_compact(c, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_row_shard(int64_t M, int world, int rank, int64_t* first_row_out, int64_t* rows_out) {
    if (M < 1 || world < 1 || rank < 0 || rank >= world || first_row_out == nullptr || rows_out == nullptr)
        return SPDP_ERR_INVALID_ARG;
    const int64_t tiles = (M + kTileM - 1) / kTileM;
    const int64_t base = tiles / world, extra = tiles % world;
    const int64_t first_tile = rank * base + (rank < extra ? rank : extra);
    const int64_t my_tiles = base + (rank < extra ? 1 : 0);
    const int64_t first = first_tile * kTileM;
    int64_t last = (first_tile + my_tiles) * kTileM;
    if (last > M) last = M;
    *first_row_out = first < M ? first : M;
    *rows_out = last > first ? last - first : 0;
    return SPDP_OK;
}

spdp_status spdp_free(spdp_handle h) {
    if (h == nullptr) {                     // no handle: give back the memory that freed handles left
        give_back_all();
        give_back_pack_totals();
        return SPDP_OK;
    }
    if (!valid(h)) return SPDP_ERR_INVALID_ARG;
    release(h);
    return SPDP_OK;
}

spdp_status spdp_get_info(spdp_handle h, spdp_info* out) {
    if (!valid(h) || out == nullptr) return SPDP_ERR_INVALID_ARG;
    spdp_info i;
    std::memset(&i, 0, sizeof(i));
    i.M = h->M; i.K = h->K; i.R = h->R; i.C = h->C; i.NGT = h->NGT;
    i.pad_elems = h->pad_elems;
    i.nnz = h->nnz;
    i.values_len = h->values_len;
    i.packed_bytes = (h->NGT + 1) * 4 + h->NGT * kTileK * 4 + h->NGT * kTileK * kWordsPerCol * 8 +
                     (h->q4 ? h->values_len / 2 + h->NGT * kTileK * 2 : h->values_len * 2);
    i.workspace_bytes = h->workspace_bytes;
    i.tileoffset_dev = h->tileoffset;
    i.colinfo_dev = h->colinfo;
    i.bitmap_dev = h->bitmap;
    i.values_dev = h->values;
    i.num_ctas = h->num_ctas;
    i.device = h->device;
    *out = i;
    return SPDP_OK;
}

spdp_status spdp_export(spdp_handle h, void* tileoffset_host, void* colinfo_host, void* bitmap_host,
                        void* values_host) {
    if (!valid(h)) return SPDP_ERR_INVALID_ARG;
    if (h->q4) return SPDP_ERR_UNSUPPORTED_SHAPE;           // 4-bit handles: spdp_export_q4
    SPDP_CUDA_TRY(cudaDeviceSynchronize());
    if (tileoffset_host)
        SPDP_CUDA_TRY(cudaMemcpy(tileoffset_host, h->tileoffset, (h->NGT + 1) * sizeof(uint32_t), cudaMemcpyDeviceToHost));
    if (colinfo_host)
        SPDP_CUDA_TRY(cudaMemcpy(colinfo_host, h->colinfo, h->NGT * kTileK * sizeof(uint32_t), cudaMemcpyDeviceToHost));
    if (bitmap_host)
        SPDP_CUDA_TRY(cudaMemcpy(bitmap_host, h->bitmap, h->NGT * kTileK * kWordsPerCol * sizeof(uint64_t),
                                 cudaMemcpyDeviceToHost));
    if (values_host && h->values_len > 0)
        SPDP_CUDA_TRY(cudaMemcpy(values_host, h->values, h->values_len * sizeof(__half), cudaMemcpyDeviceToHost));
    return SPDP_OK;
}

spdp_status spdp_unpack(spdp_handle h, void* W_dev_out, int64_t ldw, void* stream) {
    if (!valid(h) || W_dev_out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (ldw < h->K || h->q4) return SPDP_ERR_UNSUPPORTED_SHAPE;
    return unpack_device(h, static_cast<__half*>(W_dev_out), ldw, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_active_columns(spdp_handle h, const void* x_dev, spdp_dp_rule rule, float thr,
                                const void* mask_dev, void* bitmask_dev_out, void* count_dev_out,
                                void* stream) {
    if (!valid(h) || x_dev == nullptr || bitmask_dev_out == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!rule_ok(rule) || (rule == SPDP_DP_MASK && mask_dev == nullptr)) return SPDP_ERR_INVALID_ARG;
    return launch_active_columns(h, static_cast<const __half*>(x_dev), rule, thr,
                                 static_cast<const uint32_t*>(mask_dev), static_cast<uint32_t*>(bitmask_dev_out),
                                 static_cast<int*>(count_dev_out), static_cast<cudaStream_t>(stream));
}

spdp_status spdp_probe_stream_read(spdp_handle h, void* stream) {
    if (!valid(h)) return SPDP_ERR_INVALID_ARG;
    return launch_probe_stream_read(h, static_cast<cudaStream_t>(stream));
}

spdp_status spdp_probe_gather(spdp_handle h, const void* x_dev, spdp_dp_rule rule, float thr, const void* mask_dev,
                              void* stream) {
    if (!valid(h) || x_dev == nullptr) return SPDP_ERR_INVALID_ARG;
    if (!rule_ok(rule) || (rule == SPDP_DP_MASK && mask_dev == nullptr)) return SPDP_ERR_INVALID_ARG;
    if (h->pad_elems != 8) return SPDP_ERR_UNSUPPORTED_SHAPE;
    return launch_probe_gather(h, static_cast<const __half*>(x_dev), rule, thr, static_cast<const uint32_t*>(mask_dev),
                               static_cast<cudaStream_t>(stream));
}

spdp_status spdp_last_device_status(spdp_handle h, int* out) {
    if (!valid(h) || out == nullptr) return SPDP_ERR_INVALID_ARG;
    int v = 0;
    SPDP_CUDA_TRY(cudaDeviceSynchronize());
    SPDP_CUDA_TRY(cudaMemcpy(&v, h->status_word, sizeof(int), cudaMemcpyDeviceToHost));
    SPDP_CUDA_TRY(cudaMemset(h->status_word, 0, sizeof(int)));
    *out = v;
    return SPDP_OK;
}

spdp_status spdp_set_num_ctas(spdp_handle h, int num_ctas) {
    if (!valid(h) || num_ctas < 0) return SPDP_ERR_INVALID_ARG;
    DeviceScope on(h->device);
    SPDP_CUDA_TRY(cudaDeviceSynchronize());
    const spdp_status st = build_partition(h, num_ctas, nullptr);
    if (st != SPDP_OK) return st;
    SPDP_CUDA_TRY(cudaStreamSynchronize(nullptr));
    return SPDP_OK;
}

const char* spdp_last_cuda_error(void) { return g_cuda_error; }

const char* spdp_status_string(spdp_status s) {
    switch (s) {
        case SPDP_OK: return "SPDP_OK";
        case SPDP_ERR_INVALID_ARG: return "SPDP_ERR_INVALID_ARG";
        case SPDP_ERR_UNSUPPORTED_SHAPE: return "SPDP_ERR_UNSUPPORTED_SHAPE";
        case SPDP_ERR_ALLOC: return "SPDP_ERR_ALLOC";
        case SPDP_ERR_CUDA: return "SPDP_ERR_CUDA";
        case SPDP_ERR_OVERFLOW: return "SPDP_ERR_OVERFLOW";
        case SPDP_ERR_TIMEOUT: return "SPDP_ERR_TIMEOUT";
    }
    return "SPDP_ERR_UNKNOWN";
}

}  // extern "C"
