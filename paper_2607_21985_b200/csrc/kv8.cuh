// What the kernels of the 8-bit key/value cache share: its layout, what a request asks for, and how partial sums of an attention
// become its result.
//
// A cell is 16 tokens of one key head: codes of the keys [D/64][16 tokens][64 dimensions], codes of the values, the two scales.  Both
// sides lie as the fragments of a matrix product want them, so that a warp's 16-byte loads of either run through memory and what a
// lane gets needs no exchange: of the keys, lane (g, c) = (lane / 4, lane % 4) gets 16 dimensions from 16 c of token g or g + 8; of
// the values, a 32-bit word is tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9 of one dimension, and the four words of 16 bytes are
// dimensions g, g + 8, g + 16, g + 24 of 32.
#pragma once

#include "mma_f16.cuh"
#include "spdp_internal.h"

namespace spdp {
namespace kv8 {

constexpr int kCell = 16;                                                       // tokens
__host__ __device__ constexpr int cell_bytes(int dim) { return 2 * kCell * dim + 16; }
__host__ __device__ constexpr int value_place(int r, int d) {                   // byte, from the first of the values' codes
    return 512 * (d / 32) + 64 * (d % 8) + 16 * (r % 8 / 2) + 4 * (d % 32 / 8) + 2 * (r / 8) + r % 2;
}

constexpr float kLowest = -1.0e30f;     // stands for "no score yet"

struct AttnParams {
    const __half* q;
    const unsigned char* cache;
    const int32_t* table;
    const int32_t* first;               // null: one token to a request
    const int32_t* length;
    __half* y;
    uint32_t* mask;
    float* sums;                        // [2 CTAs][rows][dim]
    float2* stats;                      // [2 CTAs][rows]: maximum, weight
    int4* open;                         // triples that several CTAs have: request (-1: none), head and row block, slot of the first sum, last CTA
    bool by_triple;                     // a place of `open` for each triple; else for each CTA, of the triple that begins there
    int64_t ldq, ldy, table_stride, mask_stride;
    unsigned pages;
    int N, B, heads, group, cells_shift, most_cells;    // cells of a page: 2^cells_shift; of the longest request
    int most_blocks;                    // row blocks of a key head that a request may have
    int low_rows, most_rows;            // of a key head: requests with fewer or more are another kernel's
    int window, sinks;                  // window 0: none
    float scale, cap, cap_inv, cap_near;                // scores in powers of two; 1 / cap, and a quarter of the cap
    float thr;
    bool wide_q, wide_y;
};

// A request: its tokens n0 .. n0 + n - 1, its keys, and the cells with keys that any of its tokens sees, as one line: `sink_cells`
// from the first key on, then those from low_cell on.
struct Request {
    int n0, n, length, sink_cells, low_cell, cells;
    __device__ __forceinline__ int cell_at(int i) const { return i < sink_cells ? i : i - sink_cells + low_cell; }
};
__device__ __forceinline__ int clamped(int v, int most) { return v < 0 ? 0 : v < most ? v : most; }
__device__ __forceinline__ Request request_of(const AttnParams& p, int b) {
    Request r;
    r.n0 = b, r.n = 1;
    if (p.first != nullptr) {
        r.n0 = clamped(p.first[b], p.N);
        r.n = max(0, clamped(p.first[b + 1], p.N) - r.n0);
    }
    r.length = clamped(p.length[b], p.most_cells * kCell);
    r.low_cell = r.sink_cells = 0;
    if (p.window > 0) {
        const int at = max(r.length - r.n, 0) + 1 - p.window;                   // of the first token, whose window begins first
        r.low_cell = max(at, 0) / kCell;
        r.sink_cells = min((p.sinks + kCell - 1) / kCell, r.low_cell);
    }
    r.cells = r.n > 0 && r.length > 0 ? r.sink_cells + (r.length + kCell - 1) / kCell - r.low_cell : 0;
    const int rows = r.n * p.group;
    if (rows < p.low_rows || rows > p.most_rows) r.n = r.cells = 0;
    return r;
}
__device__ __forceinline__ bool sees(const AttnParams& p, int position, int key) {
    return key <= position && (p.window == 0 || key > position - p.window || key < p.sinks);
}

__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The two codes of a word's lower or upper half as fp16 numbers, exactly.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) {
    uint32_t r;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t high_codes(uint32_t w) {
    uint32_t r;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(w));
    return r;
}

// cap * tanh(s / cap): up to a quarter of the cap by the series of tanh, which is off by 2^-21 of s (most of it where it is cut off)
// however large the cap is; beyond, as 1 - 2 / (e^2x + 1), which keeps its limits and is off by 2^-21 of the cap, 2^-19 of s.
__device__ __forceinline__ float capped_near(const AttnParams& p, float s) {
    const float x = s * p.cap_inv, t = x * x;
    return fmaf(s * t, fmaf(fmaf(-17.0f / 315.0f, t, 2.0f / 15.0f), t, -1.0f / 3.0f), s);
}
__device__ __forceinline__ float capped_far(const AttnParams& p, float s) {
    constexpr float kTwoLog2e = 2.8853900817779268f;
    return p.cap * (1.0f - __fdividef(2.0f, exp2_of(s * p.cap_inv * kTwoLog2e) + 1.0f));
}
__device__ __forceinline__ float capped(const AttnParams& p, float s) { return fabsf(s) <= p.cap_near ? capped_near(p, s) : capped_far(p, s); }

// Four columns of a token's output and their bits of its mask; 8 neighbouring lanes have the columns of a word.
__device__ __forceinline__ void store_result(const AttnParams& p, int n, int64_t column, float4 sum, float weight) {
    const float f[4] = {sum.x, sum.y, sum.z, sum.w};
    __half y[4];
    unsigned keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = __float2half_rn(weight > 0.0f || weight != weight ? f[i] / weight : 0.0f);
        keep |= (fabsf(__half2float(y[i])) <= p.thr ? 0u : 1u) << i;
    }
    __half* to = p.y + n * p.ldy + column;
    if (p.wide_y) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(y);
    else to[0] = y[0], to[1] = y[1], to[2] = y[2], to[3] = y[3];
    if (p.mask == nullptr) return;
    keep <<= 4 * (threadIdx.x & 7);
    const unsigned mine = 0xFFu << (threadIdx.x & 24);          // the lanes of a word come together
#pragma unroll
    for (int d = 1; d < 8; d *= 2) keep |= __shfl_xor_sync(mine, keep, d);
    if ((threadIdx.x & 7) == 0) p.mask[n * p.mask_stride + column / 32] = keep;
}

// A triple costs what its units do and, for its rows and its sums, as much as kStart more: it is that long in the line of units that
// is cut into runs.
constexpr int kStart = 6;               // spdp_attn_kv8 counts on 7 at most when it checks that a line's length fits 32 bits
__device__ __forceinline__ int triple_length(int units) { return units > 0 ? units + kStart : 0; }
__device__ __forceinline__ int run_start(int total, int ctas, int i) { return static_cast<int>(static_cast<int64_t>(total) * i / ctas); }
template <int kCells, int kRows>
__device__ __forceinline__ int line_of(const AttnParams& p, const Request& r) {    // of a request, kCells to a unit and kRows to a block
    return triple_length((r.cells + kCells - 1) / kCells) * p.heads * ((r.n * p.group + kRows - 1) / kRows);
}

// Where in the line every request begins, into shared memory (all threads; ends with a barrier).
template <int kThreads, int kCells, int kRows>
__device__ void scan_line(const AttnParams& p, int* start, int* warp_sums) {
    const int each = (p.B + kThreads - 1) / kThreads, b0 = threadIdx.x * each, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int mine = 0;
    for (int b = b0; b < b0 + each && b < p.B; ++b) mine += line_of<kCells, kRows>(p, request_of(p, b));
    int up_to = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, up_to, d);
        if (lane >= d) up_to += v;
    }
    if (lane == 31) warp_sums[w] = up_to;
    __syncthreads();
    int at = up_to - mine;
    for (int i = 0; i < w; ++i) at += warp_sums[i];
    for (int b = b0; b < b0 + each && b < p.B; ++b) {
        start[b] = at;
        at += line_of<kCells, kRows>(p, request_of(p, b));
    }
    if (b0 < p.B && b0 + each >= p.B) start[p.B] = at;
    __syncthreads();
}
// The request that place u of the line belongs to.
__device__ __forceinline__ int request_at(const int* start, int B, int u) {
    int b = 0;                                                  // the last that does not begin behind u: it has keys
    for (int lo = 0, hi = B - 1; lo <= hi;) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= u) b = mid, lo = mid + 1;
        else hi = mid - 1;
    }
    return b;
}

// Zeros for the tokens of requests without keys.
__device__ inline void store_nothing(const AttnParams& p, const Request& r, int dim, int threads) {
    const int columns = p.heads * p.group * dim;
    for (int n = r.n0; n < r.n0 + r.n; ++n) {
        for (int i = threadIdx.x; i < columns; i += threads) p.y[n * p.ldy + i] = __ushort_as_half(0);
        if (p.mask != nullptr)
            for (int i = threadIdx.x; i < columns / 32; i += threads) p.mask[n * p.mask_stride + i] = 0.0f <= p.thr ? 0u : 0xFFFFFFFFu;
    }
}

// Joins the partial sums of a triple that several CTAs have, in the order of its keys: a row of it to a CTA, whose groups of lanes
// take every kParts-th sum.
constexpr int kJoinThreads = 256;

template <int kDim, int kRows>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const AttnParams p) {
    constexpr int kLanes = kDim / 4, kParts = kJoinThreads / kLanes;
    __shared__ __align__(16) float part[kParts][kDim];
    __shared__ float2 stat[kParts];
    dev::programmatic_start();
    const int4 open = p.open[blockIdx.x];
    if (open.x < 0) return;
    const Request r = request_of(p, open.x);
    const int h = open.y / p.most_blocks, row = blockIdx.y, mine_row = open.y % p.most_blocks * kRows + row;
    if (mine_row >= r.n * p.group) return;
    const int at = threadIdx.x % kLanes, mine = threadIdx.x / kLanes, count = open.w - open.z / 2 + 1;
    float m = kLowest, wt = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int i = mine; i < count; i += kParts) {
        const int64_t from = (i == 0 ? open.z : 2 * (open.z / 2 + static_cast<int64_t>(i))) * kRows + row;
        const float2 st = p.stats[from];
        const float4 v = *reinterpret_cast<const float4*>(p.sums + from * kDim + 4 * at);
        const float top = fmaxf(m, st.x), f = exp2_of(m - top), fs = exp2_of(st.x - top);
        sum.x = sum.x * f + v.x * fs, sum.y = sum.y * f + v.y * fs, sum.z = sum.z * f + v.z * fs, sum.w = sum.w * f + v.w * fs;
        wt = wt * f + st.y * fs;
        m = top;
    }
    *reinterpret_cast<float4*>(&part[mine][4 * at]) = sum;
    if (at == 0) stat[mine] = make_float2(m, wt);
    __syncthreads();
    const int d = 4 * threadIdx.x;
    if (d >= kDim) return;
    m = kLowest, wt = 0.0f;
    sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kParts; ++i) m = fmaxf(m, stat[i].x);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const float f = exp2_of(stat[i].x - m);
        const float4 v = *reinterpret_cast<const float4*>(&part[i][d]);
        wt += stat[i].y * f;
        sum.x += v.x * f, sum.y += v.y * f, sum.z += v.z * f, sum.w += v.w * f;
    }
    store_result(p, r.n0 + mine_row / p.group, static_cast<int64_t>(h * p.group + mine_row % p.group) * kDim + d, sum, wt);
}

// The same for few triples of many sums each, where it is all latency: the first kAhead sums of a group are asked for together with
// all maxima.  Taken from kJoinFew CTAs to a triple on.  Attention and join in the form above / in this one, us, all of the GPU on 1, 8, 16 and 24 triples of 200000 keys
// together (9000 each at least): heads of 128 47 / 37, 29 / 29, 27 / 29, 27 / 29; of 256 64 / 47, 39 / 37, 37 / 37, 37 / 39; of 64 29 / 29, 21 / 23, 21 / 23, 21 / 23.
constexpr int kJoinFew = 16;
constexpr int kJoinChunk = kJoinThreads;                        // sums whose maxima and weights are in shared memory at a time

template <int kDim, int kRows>
__global__ void __launch_bounds__(kJoinThreads) attn_join_few_kernel(const AttnParams p) {
    constexpr int kLanes = kDim / 4, kParts = kJoinThreads / kLanes, kAhead = 12;
    __shared__ __align__(16) float part[kParts][kDim];
    __shared__ float2 stats[kJoinChunk];
    __shared__ float warp_tops[kJoinThreads / 32], weights[kParts];
    dev::programmatic_start();
    const int4 open = p.open[blockIdx.x];
    if (open.x < 0) return;
    const Request r = request_of(p, open.x);
    const int h = open.y / p.most_blocks, row = blockIdx.y, mine_row = open.y % p.most_blocks * kRows + row;
    if (mine_row >= r.n * p.group) return;
    const int at = threadIdx.x % kLanes, mine = threadIdx.x / kLanes, count = open.w - open.z / 2 + 1;
    auto place = [&](int i) { return (i == 0 ? open.z : 2 * (open.z / 2 + static_cast<int64_t>(i))) * kRows + row; };
    auto sum_at = [&](int i) { return *reinterpret_cast<const float4*>(p.sums + place(i) * kDim + 4 * at); };
    float4 ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (mine + j * kParts < count) ahead[j] = sum_at(mine + j * kParts);
    float m = kLowest, wt = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [&](float4 v, float2 st) {
        const float f = exp2_of(st.x - m);
        sum.x += v.x * f, sum.y += v.y * f, sum.z += v.z * f, sum.w += v.w * f;
        wt += st.y * f;
    };
    for (int i0 = 0; i0 < count; i0 += kJoinChunk) {
        const int n = min(kJoinChunk, count - i0);
        float top = m;
        for (int i = threadIdx.x; i < n; i += kJoinThreads) {
            stats[i] = p.stats[place(i0 + i)];
            top = fmaxf(top, stats[i].x);
        }
#pragma unroll
        for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        if (threadIdx.x % 32 == 0) warp_tops[threadIdx.x / 32] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kJoinThreads / 32; ++i) top = fmaxf(top, warp_tops[i]);
        const float f = exp2_of(m - top);
        sum.x *= f, sum.y *= f, sum.z *= f, sum.w *= f, wt *= f, m = top;
        int i = mine;
        if (i0 == 0) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j, i += kParts)
                if (i < n) add(ahead[j], stats[i]);
        }
#pragma unroll 4
        for (; i < n; i += kParts) add(sum_at(i0 + i), stats[i]);
        __syncthreads();                                        // before the next maxima take their place
    }
    *reinterpret_cast<float4*>(&part[mine][4 * at]) = sum;
    if (at == 0) weights[mine] = wt;
    __syncthreads();
    const int d = 4 * threadIdx.x;
    if (d >= kDim) return;
    wt = 0.0f;
    sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const float4 v = *reinterpret_cast<const float4*>(&part[i][d]);
        wt += weights[i];
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
    store_result(p, r.n0 + mine_row / p.group, static_cast<int64_t>(h * p.group + mine_row % p.group) * kDim + d, sum, wt);
}

}  // namespace kv8

// kv8_prompt.cu: the requests with a.low_rows rows and more.
spdp_status launch_kv8_prompt(const kv8::AttnParams& a, int head_dim, int device, int sms, cudaStream_t s);

}  // namespace spdp
