// A paged key/value cache of 8-bit codes with a scale to every 16 tokens of a head (kv8.cuh has its layout): storing rows, and the
// attention of requests with few new tokens over it.  kv8_prompt.cu has the attention of longer pieces of prompts.
#include <cooperative_groups.h>

#include <cfloat>
#include <mutex>

#include "kv8.cuh"

namespace cg = cooperative_groups;

namespace spdp {
namespace {

using namespace kv8;

// ---- storing ----------------------------------------------------------------------------------------------------------------
//
// A warp takes one side (keys or values) of one cell: it has all its new tokens at once, so the scale needs one reduction within the
// warp and no atomics, and a cell that grows is rounded again by the warp that makes it grow.  Scales are powers of two: dividing
// by one is exact, so a code is rounded once, and what it stands for is an fp16 number; and a code that is rounded again for
// a larger scale stays what it was unless it is a small one.
// What bounds it: issue (54 % of the slots: conversions, the values' transposes) and one load's wait after another (starts, length, table, rows).
// 16384 tokens of 8 heads of 128, 32-bit values, all written back as fp16: 41 us, 201 MB at 4.9 TB/s, of which 157 MB reach memory.

constexpr int kStoreWarps = 4;
constexpr float kMost = 61440.0f;       // 240 * 2^8, the largest that a code can stand for within fp16

struct StoreParams {
    const __half* k;
    const void* v;
    const int32_t* table;
    const int32_t* first;               // null: one token to a request
    const int32_t* length;
    unsigned char* cache;
    __half* k_values;
    __half* v_values;
    int64_t ldk, ldv, ldk_values, ldv_values, table_stride, items;
    unsigned pages;
    int N, B, heads, cells_shift, most_cells, chunk;    // a warp looks for cells that begin in `chunk` tokens
};

// The last of B requests whose tokens begin at n or before it: all lanes look at once.
__device__ __forceinline__ int request_of_token(const int32_t* first, int B, int n) {
    const int lane = threadIdx.x & 31;
    int low = 0, count = B;                                     // among `low` .. low + count - 1; low's tokens begin at n or before it (or there is none such)
    while (count > 1) {
        const int step = (count + 31) / 32, at = low + lane * step;
        const bool before = lane * step < count && first[at] <= n;
        const unsigned found = __ballot_sync(0xFFFFFFFFu, before);
        const int last = found == 0u ? 0 : 31 - __clz(found);
        const int end = low + count;
        low += last * step;
        count = min(step, end - low);
        if (found == 0u) count = 1;
    }
    return low;
}

// The smallest 2^e with top <= 448 * 2^e, e >= -15.
__device__ __forceinline__ float scale_for(float top) {
    const uint32_t bits = __float_as_uint(top);
    const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float(static_cast<uint32_t>(max(e, -15) + 127) << 23);
}
// Four fp16 numbers, times a power of two, to codes.
__device__ __forceinline__ uint32_t codes_of(uint2 x, __half2 factor) {
    uint32_t r;
    const __half2 a = __hmul2(*reinterpret_cast<const __half2*>(&x.x), factor), b = __hmul2(*reinterpret_cast<const __half2*>(&x.y), factor);
    asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f16x2 l, %1;\n cvt.rn.satfinite.e4m3x2.f16x2 h, %2;\n mov.b32 %0, {l, h};\n}"
        : "=r"(r) : "r"(*reinterpret_cast<const uint32_t*>(&a)), "r"(*reinterpret_cast<const uint32_t*>(&b)));
    return r;
}
__device__ __forceinline__ uint2 halves_of(uint32_t codes, __half2 factor) {
    const uint32_t a = low_codes(codes), b = high_codes(codes);
    const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&a), factor), y = __hmul2(*reinterpret_cast<const __half2*>(&b), factor);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
}
// Codes rounded again for a scale 1 / ratio times theirs.
__device__ __forceinline__ uint32_t again(uint32_t codes, __half2 ratio) { return codes_of(halves_of(codes, ratio), __half2half2(__ushort_as_half(0x3C00))); }

// Bytes i of a, b, c, d become the word out[i].
__device__ __forceinline__ void transpose_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4]) {
    const uint32_t ab_low = __byte_perm(a, b, 0x5140), ab_high = __byte_perm(a, b, 0x7362), cd_low = __byte_perm(c, d, 0x5140), cd_high = __byte_perm(c, d, 0x7362);
    out[0] = __byte_perm(ab_low, cd_low, 0x5410), out[1] = __byte_perm(ab_low, cd_low, 0x7632);
    out[2] = __byte_perm(ab_high, cd_high, 0x5410), out[3] = __byte_perm(ab_high, cd_high, 0x7632);
}
// Of the lanes that differ in the bits `near` and `far`: lane i of four gets the words i of all of them, in their order.
__device__ __forceinline__ uint4 transpose_words(uint32_t a, uint32_t b, uint32_t c, uint32_t d, int near, int far) {
    const int lane = threadIdx.x & 31;
    const bool odd = lane & near, high = lane & far;
    uint32_t x = __shfl_xor_sync(0xFFFFFFFFu, odd ? a : b, near), y = __shfl_xor_sync(0xFFFFFFFFu, odd ? c : d, near);
    if (odd) a = x, c = y;
    else b = x, d = y;
    x = __shfl_xor_sync(0xFFFFFFFFu, high ? a : c, far), y = __shfl_xor_sync(0xFFFFFFFFu, high ? b : d, far);
    if (high) a = x, b = y;
    else c = x, d = y;
    return make_uint4(a, b, c, d);
}

// Four values of a row, as they are.
template <typename T> struct Four { uint2 v; };
template <> struct Four<float> { uint4 v; };
template <typename T, bool kWide>
__device__ __forceinline__ Four<T> load_four(const T* at) {
    Four<T> r;
    if constexpr (sizeof(T) == 2) {
        const unsigned short* u = reinterpret_cast<const unsigned short*>(at);
        if constexpr (kWide) r.v = *reinterpret_cast<const uint2*>(at);
        else r.v = make_uint2(u[0] | static_cast<uint32_t>(u[1]) << 16, u[2] | static_cast<uint32_t>(u[3]) << 16);
    } else {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(at);
        if constexpr (kWide) r.v = *reinterpret_cast<const uint4*>(at);
        else r.v = make_uint4(u[0], u[1], u[2], u[3]);
    }
    return r;
}
template <bool kWide>
__device__ __forceinline__ void store_four(__half* at, uint2 h) {
    if constexpr (kWide) *reinterpret_cast<uint2*>(at) = h;
    else {
        unsigned short* u = reinterpret_cast<unsigned short*>(at);
        u[0] = static_cast<unsigned short>(h.x), u[1] = static_cast<unsigned short>(h.x >> 16), u[2] = static_cast<unsigned short>(h.y), u[3] = static_cast<unsigned short>(h.y >> 16);
    }
}
// The same as fp16 numbers within the cache's range.
template <typename T>
__device__ __forceinline__ uint2 limited(const Four<T>& x) {
    __half2 a, b;
    if constexpr (sizeof(T) == 2) a = *reinterpret_cast<const __half2*>(&x.v.x), b = *reinterpret_cast<const __half2*>(&x.v.y);
    else {
        a = __floats2half2_rn(__uint_as_float(x.v.x), __uint_as_float(x.v.y));
        b = __floats2half2_rn(__uint_as_float(x.v.z), __uint_as_float(x.v.w));
    }
    const __half2 top = __float2half2_rn(kMost), bottom = __float2half2_rn(-kMost);
    a = __hmax2(__hmin2(a, top), bottom), b = __hmax2(__hmin2(b, top), bottom);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// One side of a cell, whose tokens old .. end - 1 are new (those before have been there, those behind do not exist): token r of the cell is row `row0`
// + r of x.  cell: null where there is none to store to.  A lane has 4 dimensions (of 128 at a time) of all 16 tokens or,
// with 64 dimensions, of half of them: tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9 for its values of t, as the values' words have them.
template <typename T, int kDim, bool kWide>
__device__ __forceinline__ void store_side(const T* x, int64_t ld, __half* values, int64_t ld_values, int64_t row0, int old, int end, unsigned char* cell, bool is_v) {
    constexpr int kLanes = kDim == 64 ? 16 : 32, kTs = 4 * kLanes / 32, kLoops = kDim > 128 ? kDim / 128 : 1;
    const int lane = threadIdx.x & 31, part = lane / kLanes, d0 = 4 * (lane % kLanes);
    auto token = [&](int t, int i) { return 2 * (part * kTs + t) + (i & 1) + 8 * (i >> 1); };
    if (end == old + 1 && old > 0 && cell != nullptr) {         // one token behind others, whose scale is usually large enough: only its own bytes
        const float scale = *reinterpret_cast<const float*>(cell + 2 * kCell * kDim + (is_v ? 4 : 0));
        uint2 f[kLoops];
        __half2 most = __float2half2_rn(0.0f);
#pragma unroll
        for (int l = 0; l < kLoops; ++l) {
            f[l] = limited<T>(load_four<T, kWide>(x + (row0 + old) * ld + 128 * l + d0));
            most = __hmax2(most, __hmax2(__habs2(*reinterpret_cast<const __half2*>(&f[l].x)), __habs2(*reinterpret_cast<const __half2*>(&f[l].y))));
        }
        const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, max(static_cast<uint32_t>(__half_as_ushort(__low2half(most))), static_cast<uint32_t>(__half_as_ushort(__high2half(most)))));
        if (scale_for(__half2float(__ushort_as_half(static_cast<unsigned short>(bits)))) <= scale) {
            if (part > 0) return;                               // the other half of the warp has the same dimensions
#pragma unroll
            for (int l = 0; l < kLoops; ++l) {
                const int d = 128 * l + d0;
                const uint32_t c = codes_of(f[l], __float2half2_rn(1.0f / scale));
                if (!is_v) *reinterpret_cast<uint32_t*>(cell + d / 64 * 1024 + old * 64 + d % 64) = c;
                else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) cell[kCell * kDim + value_place(old, d + j)] = static_cast<unsigned char>(c >> 8 * j);
                }
                if (values != nullptr) store_four<kWide>(values + (row0 + old) * ld_values + d, halves_of(c, __float2half2_rn(scale)));
            }
            return;
        }
    }
    uint2 f[kLoops][kTs][4];
    __half2 most = __float2half2_rn(0.0f);
    float scale_old = 0.0f;
    if (old > 0 && cell != nullptr) scale_old = *reinterpret_cast<const float*>(cell + 2 * kCell * kDim + (is_v ? 4 : 0));
#pragma unroll
    for (int l = 0; l < kLoops; ++l) {
        Four<T> raw[kTs][4];                                    // all on their way before the first is looked at
#pragma unroll
        for (int t = 0; t < kTs; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = token(t, i);
                raw[t][i] = {};
                if (r >= old && r < end) raw[t][i] = load_four<T, kWide>(x + (row0 + r) * ld + 128 * l + d0);
            }
        }
#pragma unroll
        for (int t = 0; t < kTs; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[l][t][i] = limited<T>(raw[t][i]);
        }
    }
#pragma unroll
    for (int l = 0; l < kLoops; ++l) {
#pragma unroll
        for (int t = 0; t < kTs; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                most = __hmax2(most, __hmax2(__habs2(*reinterpret_cast<const __half2*>(&f[l][t][i].x)), __habs2(*reinterpret_cast<const __half2*>(&f[l][t][i].y))));
        }
    }
    // the bits of numbers from 0 up are in their order
    const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, max(static_cast<uint32_t>(__half_as_ushort(__low2half(most))), static_cast<uint32_t>(__half_as_ushort(__high2half(most)))));
    const float need = scale_for(__half2float(__ushort_as_half(static_cast<unsigned short>(bits))));
    const float scale = fmaxf(need, scale_old);
    const bool grows = scale > scale_old && old > 0 && cell != nullptr;
    const __half2 up = __float2half2_rn(scale), down = __float2half2_rn(1.0f / scale), ratio = __float2half2_rn(scale_old / scale);
    if (cell != nullptr && lane == 0 && (scale > scale_old || old == 0)) *reinterpret_cast<float*>(cell + 2 * kCell * kDim + (is_v ? 4 : 0)) = scale;
    if (cell != nullptr && lane < 2 && old == 0 && is_v) *reinterpret_cast<float*>(cell + 2 * kCell * kDim + 8 + 4 * lane) = 0.0f;
    unsigned char* codes = cell + (is_v ? kCell * kDim : 0);
#pragma unroll
    for (int l = 0; l < kLoops; ++l) {
        uint32_t c[kTs][4];
#pragma unroll
        for (int t = 0; t < kTs; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = token(t, i);
                c[t][i] = codes_of(f[l][t][i], down);
                if (values != nullptr && r >= old && r < end) {
                    store_four<kWide>(values + (row0 + r) * ld_values + 128 * l + d0, halves_of(c[t][i], up));
                }
            }
        }
        if (cell == nullptr) continue;
        if (!is_v) {
            const int d = 128 * l + d0;
#pragma unroll
            for (int t = 0; t < kTs; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = token(t, i);
                    uint32_t* to = reinterpret_cast<uint32_t*>(codes + d / 64 * 1024 + r * 64 + d % 64);
                    if (r < old) {
                        if (grows) *to = again(*to, ratio);
                    } else if (r < end || old == 0) *to = c[t][i];
                }
            }
            continue;
        }
        // words of four tokens of a dimension, then the words of dimensions d, d + 8, d + 16, d + 24 (of lanes i, i + 2, i + 4, i + 6) together
        uint32_t w[4][4];                                       // [dimension of the lane's][t]
#pragma unroll
        for (int t = 0; t < kTs; ++t) {
            uint32_t o[4];
            transpose_bytes(c[t][0], c[t][1], c[t][2], c[t][3], o);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j][t] = o[j];
        }
        if constexpr (kTs == 2) {                               // the other half of the warp has the other two t: two dimensions each
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t a = __shfl_xor_sync(0xFFFFFFFFu, part ? w[0][t] : w[2][t], 16), b = __shfl_xor_sync(0xFFFFFFFFu, part ? w[1][t] : w[3][t], 16);
                if (part) w[0][2 + t] = w[2][t], w[1][2 + t] = w[3][t], w[0][t] = a, w[1][t] = b;
                else w[0][2 + t] = a, w[1][2 + t] = b;
            }
        }
        const int t = lane >> 1 & 3;
        unsigned known = 0, fresh = 0;                          // bytes of the lane's words: tokens that have been there, and new ones
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 2 * t + (i & 1) + 8 * (i >> 1);
            if (r < old) known |= 0xFFu << 8 * i;
            else if (r < end) fresh |= 0xFFu << 8 * i;
        }
#pragma unroll
        for (int j = 0; j < (kTs == 2 ? 2 : 4); ++j) {
            uint4 mine = transpose_words(w[j][0], w[j][1], w[j][2], w[j][3], 2, 4);
            const int d = 128 * l + d0 % 32 % 8 + d0 / 32 * 32 + j + (kTs == 2 ? 2 * part : 0);     // of the first of its words
            uint4* to = reinterpret_cast<uint4*>(codes + 512 * (d / 32) + 64 * (d % 8) + 16 * t);
            if (known != 0) {
                if (!grows && fresh == 0) continue;
                uint4 was = *to;
                if (grows) was = make_uint4(again(was.x, ratio), again(was.y, ratio), again(was.z, ratio), again(was.w, ratio));
                mine.x = (was.x & known) | (mine.x & ~known), mine.y = (was.y & known) | (mine.y & ~known);
                mine.z = (was.z & known) | (mine.z & ~known), mine.w = (was.w & known) | (mine.w & ~known);
            } else if (fresh == 0 && old > 0) continue;
            *to = mine;
        }
    }
}

template <typename V, int kDim, bool kWide>
__global__ void __launch_bounds__(32 * kStoreWarps) kv8_store_kernel(const StoreParams p) {
    dev::programmatic_start();
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kStoreWarps + (threadIdx.x >> 5);
    if (item >= p.items) return;
    const int h = static_cast<int>(item % p.heads);
    const bool is_v = item / p.heads % 2 != 0;
    const int64_t begin = item / p.heads / 2 * p.chunk;
    const int stop = static_cast<int>(begin + p.chunk < p.N ? begin + p.chunk : p.N), lane = threadIdx.x & 31;
    // up to 31 requests, a lane knows where one begins and how long it is: what a warp waits for one load after another, not the requests'
    // number of them, is most of its time
    const bool few = p.first != nullptr && p.B < 32;
    int lane_first = 0, lane_length = 0;
    if (few) lane_first = clamped(p.first[min(lane, p.B)], p.N), lane_length = p.length[min(lane, p.B - 1)];
    for (int n = static_cast<int>(begin); n < stop;) {
        int b = n, first = n, last = n + 1, length;             // the request's tokens: first .. last - 1
        if (few) {
            b = max(31 - __clz(__ballot_sync(0xFFFFFFFFu, lane < p.B && lane_first <= n)), 0);
            first = __shfl_sync(0xFFFFFFFFu, lane_first, b), last = __shfl_sync(0xFFFFFFFFu, lane_first, b + 1), length = __shfl_sync(0xFFFFFFFFu, lane_length, b);
        } else {
            if (p.first != nullptr) {
                b = request_of_token(p.first, p.B, n);
                first = clamped(p.first[b], p.N), last = clamped(p.first[b + 1], p.N);
            }
            length = p.length[b];
        }
        if (first > n || last <= n) {                           // a token of no request
            ++n;
            continue;
        }
        const int place = clamped(length, p.most_cells * kCell) - (last - n);          // the token's among its request's keys
        const int old = place < 0 ? place : place % kCell;
        if (old < 0 || (old > 0 && n != first)) {               // nowhere to store it, or the warp of its cell's first new token does
            n += old < 0 ? min(-old, last - n) : min(kCell - old, last - n);
            continue;
        }
        const int end = min(kCell, old + (last - n)), at = place / kCell;
        const unsigned page = p.table[b * p.table_stride + (at >> p.cells_shift)];
        unsigned char* cell = nullptr;
        if (page < p.pages)
            cell = p.cache + (((static_cast<int64_t>(page) * p.heads + h) << p.cells_shift) + (at & ((1 << p.cells_shift) - 1))) * cell_bytes(kDim);
        const int64_t row0 = static_cast<int64_t>(n) - old;
        if (is_v) store_side<V, kDim, kWide>(static_cast<const V*>(p.v) + h * kDim, p.ldv, p.v_values != nullptr ? p.v_values + h * kDim : nullptr, p.ldv_values, row0, old, end, cell, true);
        else store_side<__half, kDim, kWide>(p.k + h * kDim, p.ldk, p.k_values != nullptr ? p.k_values + h * kDim : nullptr, p.ldk_values, row0, old, end, cell, false);
        n += end - old;
    }
}

template <typename V, int kDim>
cudaError_t launch_store(StoreParams p, bool wide, int sms, cudaStream_t s) {
    // a warp to each token's cell where that leaves SMs idle, else one to 16 tokens
    const int64_t sides = 2 * static_cast<int64_t>(p.heads);
    p.chunk = p.first != nullptr && (p.N + kCell - 1) / kCell * sides > 4 * sms ? kCell : 1;
    p.items = (p.N + p.chunk - 1) / p.chunk * sides;
    const dim3 grid(static_cast<unsigned>((p.items + kStoreWarps - 1) / kStoreWarps));
    return launch_programmatic(wide ? kv8_store_kernel<V, kDim, true> : kv8_store_kernel<V, kDim, false>, grid, 32 * kStoreWarps, 0, s, p);
}

// ---- attention of few tokens ------------------------------------------------------------------------------------------------
//
// The rows of a (request, key head) are its tokens' query heads, token by token; kRows of them are a triple's.  The keys of all triples,
// 64 to a unit, stand in one line that is cut into equal runs, one to a CTA: so one long request and many short ones alike
// occupy the whole GPU, whatever the lengths are, which only the device knows.  A run that holds a triple's every key writes its
// output; else CTAs leave a partial sum of it, with its maximum and its weight, and a second kernel joins them in the order
// of the keys.
//
// Scores are K q^T and outputs V^T P^T on mma.sync with the rows as the 8 columns, from registers to registers: a cell is 2 D
// fragments of 16 bytes, which the next step's loads bring while this step's are worked on.  Codes enter the products as the
// fp16 numbers they are.  The keys' scale multiplies the scores, the values' scale 2^e the weights: as a term of the exponent, so
// that what is rounded to fp16 (2^-11, the one rounding besides the result's) is as large as it counts in the sum.
// What bounds it: memory.  48 requests of up to 16384 keys, 64 and 8 heads of 128: 890 MB in 143 us (6.2 TB/s); one request of 131072: 271 MB in 51.5 us
// (5.3 TB/s), the start and the end of a run being 4 us of it.  Issue is 33 to 39 % busy: a cell is 64 conversions (two codes each), 16 products.  Rows behind
// the first 8 or 16 go through the keys again, and that is not hidden behind the bytes: one request of 131072 keys takes 76 us with 16 rows, 127 with 32, 226 with 64.

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kUnitCells = 4;
constexpr int kMostRequests = 4096;
constexpr float kHeadroom = 12.0f;      // weights are below 2^(kHeadroom + kSlack)
constexpr float kSlack = 2.5f;

template <int kChunks, int kCols>
struct Shape {
    static constexpr int kDim = 64 * kChunks, kRows = 8 * kCols;
    static constexpr int kCells = kChunks * kCols <= 2 ? 2 : 1;         // of a step
    static constexpr int kCtasOfSm = kChunks == 4 ? 2 : kChunks * kCols == 1 ? 4 : 3;  // that the registers are cut for
    static constexpr int kSums = kRows * kDim * 4;                      // bytes of a warp's sums
};

__device__ __forceinline__ uint4 load16(const unsigned char* at) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(at));
    return v;
}
__device__ __forceinline__ float2 load_scales(const unsigned char* at) {
    float2 v;
    asm volatile("ld.global.L1::no_allocate.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(at));
    return v;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// A CTA's warps over the cells c0 .. c1 - 1 of a triple's line: a warp's sums [kRows][kDim] end up in its part of `sums`, its maxima
// and weights in warp_stats [warp][kRows].
template <int kChunks, int kCols>
__device__ __forceinline__ void attend(const AttnParams& p, const Request& rq, int b, int h, int row0, int c0, int c1, unsigned char* sums, float2* warp_stats) {
    using S = Shape<kChunks, kCols>;
    constexpr int kDim = S::kDim, kRows = S::kRows, kCells = S::kCells, kLoads = 2 * kChunks;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int rows = min(kRows, rq.n * p.group - row0), before = rq.length - rq.n;      // keys before the request's first token
    const int32_t* table = p.table + b * p.table_stride;
    const unsigned char* const head = p.cache + (static_cast<int64_t>(h) << p.cells_shift) * cell_bytes(kDim) + 16 * lane;
    const int64_t page_bytes = (static_cast<int64_t>(p.heads) << p.cells_shift) * cell_bytes(kDim);
    const int in_page = (1 << p.cells_shift) - 1;

    // The warp's steps: every fourth one of the run.  Each lane knows the page of a cell of the next 32 / kCells of them.
    const int steps = ((c1 - c0 + kCells - 1) / kCells - w + kWarps - 1) / kWarps;
    constexpr int kAhead = 32 / kCells;
    auto cell_of = [&](int i, int j) { return c0 + kCells * (w + kWarps * i) + j; };
    auto pages_of = [&](int i) {
        const int at = cell_of(i + lane / kCells, lane % kCells);
        return at < c1 ? table[rq.cell_at(at) >> p.cells_shift] : -1;
    };
    int pages = pages_of(0), pages_after = pages_of(kAhead);
    uint4 k[kCells][kLoads], v[kCells][kLoads];
    float2 scales[kCells], scales_next[kCells];
    bool there[kCells], there_next[kCells];
    const unsigned char* at_next[kCells];
    auto locate = [&](int i) {                                  // where the cells of step i are
        if (i > 0 && i % kAhead == 0) pages = pages_after, pages_after = pages_of(i + kAhead);
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
            const unsigned page = __shfl_sync(0xFFFFFFFFu, pages, (i * kCells + j) & 31);
            there_next[j] = i < steps && page < p.pages;        // negative ones are large here
            at_next[j] = head + static_cast<int64_t>(there_next[j] ? page : 0u) * page_bytes + (rq.cell_at(cell_of(i, j)) & in_page) * cell_bytes(kDim);
        }
    };
    auto load_keys = [&]() {
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
            scales_next[j] = make_float2(0.0f, 1.0f);
            if (there_next[j]) scales_next[j] = load_scales(at_next[j] + 2 * kCell * kDim - 16 * lane);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                k[j][i] = make_uint4(0, 0, 0, 0);
                if (there_next[j]) k[j][i] = load16(at_next[j] + 512 * i);
            }
        }
    };
    auto load_values = [&]() {
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                v[j][i] = make_uint4(0, 0, 0, 0);
                if (there_next[j]) v[j][i] = load16(at_next[j] + kCell * kDim + 512 * i);
            }
        }
    };
    locate(0);
    load_keys();
    load_values();

    // the rows as the products' columns
    uint32_t q[kCols][4 * kChunks][2];
    int position[kCols][2];                                     // of the columns 2 c and 2 c + 1
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
        const int row = row0 + min(8 * n + g, rows - 1);        // columns behind the last are copies of it
        const __half* at = p.q + (rq.n0 + row / p.group) * p.ldq + static_cast<int64_t>(h * p.group + row % p.group) * kDim + 16 * c;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            uint32_t x[8];
            if (p.wide_q) {
                const uint4 a = *reinterpret_cast<const uint4*>(at + 64 * i), d = *reinterpret_cast<const uint4*>(at + 64 * i + 8);
                x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = d.x, x[5] = d.y, x[6] = d.z, x[7] = d.w;
            } else {
                const unsigned short* u = reinterpret_cast<const unsigned short*>(at + 64 * i);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = u[2 * j] | static_cast<uint32_t>(u[2 * j + 1]) << 16;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) q[n][4 * i + j][0] = x[2 * j], q[n][4 * i + j][1] = x[2 * j + 1];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) position[n][i] = before + (row0 + min(8 * n + 2 * c + i, rows - 1)) / p.group;
    }
    const int earliest = before + row0 / p.group, latest = before + (row0 + rows - 1) / p.group;

    float acc[kCols][4 * kChunks][4] = {};
    float top[kCols][2], weight[kCols][2];
#pragma unroll
    for (int n = 0; n < kCols; ++n) top[n][0] = top[n][1] = kLowest, weight[n][0] = weight[n][1] = 0.0f;

    for (int i = 0; i < steps; ++i) {
        int key[kCells];
        bool whole = true;
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
            scales[j] = scales_next[j], there[j] = there_next[j];
            key[j] = rq.cell_at(cell_of(i, j)) * kCell;
            whole &= there[j] && key[j] + kCell - 1 <= earliest && (p.window == 0 || key[j] > latest - p.window || key[j] + kCell <= p.sinks);
        }
        float score[kCols][kCells][4] = {};
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
#pragma unroll
            for (int t = 0; t < kChunks; ++t) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const uint32_t x = word(k[j][2 * t], m), y = word(k[j][2 * t + 1], m);
                    const uint32_t a0 = low_codes(x), a1 = low_codes(y), a2 = high_codes(x), a3 = high_codes(y);
#pragma unroll
                    for (int n = 0; n < kCols; ++n) dev::mma_f16(score[n][j], a0, a1, a2, a3, q[n][4 * t + m][0], q[n][4 * t + m][1]);
                }
            }
        }
        locate(i + 1);
        load_keys();
        float back[kCells];                                     // 1 / the values' scale
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
            const int e = __float_as_int(scales[j].y) >> 23 & 255;
            const float up = static_cast<float>(e - 127), f = scales[j].x * p.scale;
            back[j] = __int_as_float((254 - e) << 23);
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (p.cap > 0.0f) score[n][j][m] = capped(p, score[n][j][m] * f) + up;
                    else score[n][j][m] = fmaf(score[n][j][m], f, up);
                }
            }
        }
        if (!whole) {
#pragma unroll
            for (int j = 0; j < kCells; ++j) {
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        if (!there[j] || !sees(p, position[n][m & 1], key[j] + g + 8 * (m >> 1))) score[n][j][m] = -INFINITY;
                    }
                }
                uint32_t keep = 0;                              // the values' bytes behind the last key: whatever the cell holds there
#pragma unroll
                for (int m = 0; m < 4; ++m) keep |= key[j] + 2 * c + (m & 1) + 8 * (m >> 1) <= latest ? 0xFFu << 8 * m : 0u;
#pragma unroll
                for (int t = 0; t < kLoads; ++t) v[j][t].x &= keep, v[j][t].y &= keep, v[j][t].z &= keep, v[j][t].w &= keep;
            }
        }
        // The weights are 2^(score - top), where top is the largest score so far less kHeadroom, or up to kSlack less: as large as fp16
        // allows, so that small ones keep their digits.
        bool renew = false;
        float high[kCols][2];
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                high[n][m] = fmaxf(score[n][0][m], score[n][0][2 + m]);
#pragma unroll
                for (int j = 1; j < kCells; ++j) high[n][m] = fmaxf(high[n][m], fmaxf(score[n][j][m], score[n][j][2 + m]));
                renew |= high[n][m] > top[n][m] + (kHeadroom + kSlack);
            }
        }
        if (__any_sync(0xFFFFFFFFu, renew)) {
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    float largest = high[n][m];
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) largest = fmaxf(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, d));
                    const float next = fmaxf(top[n][m], largest - kHeadroom), f = exp2_of(top[n][m] - next);
                    top[n][m] = next;
                    weight[n][m] *= f;
#pragma unroll
                    for (int t = 0; t < 4 * kChunks; ++t) acc[n][t][m] *= f, acc[n][t][2 + m] *= f;
                }
            }
        }
        uint32_t lo[kCols][kCells], hi[kCols][kCells];
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
#pragma unroll
            for (int j = 0; j < kCells; ++j) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    score[n][j][m] = exp2_of(score[n][j][m] - top[n][m & 1]);
                    weight[n][m & 1] = fmaf(score[n][j][m], back[j], weight[n][m & 1]);
                }
                const __half2 a = __floats2half2_rn(score[n][j][0], score[n][j][1]), d = __floats2half2_rn(score[n][j][2], score[n][j][3]);
                lo[n][j] = transpose8x8(*reinterpret_cast<const uint32_t*>(&a)), hi[n][j] = transpose8x8(*reinterpret_cast<const uint32_t*>(&d));
            }
        }
#pragma unroll
        for (int j = 0; j < kCells; ++j) {
#pragma unroll
            for (int t = 0; t < kLoads; ++t) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint32_t x = word(v[j][t], 2 * m), y = word(v[j][t], 2 * m + 1);
                    const uint32_t a0 = low_codes(x), a1 = low_codes(y), a2 = high_codes(x), a3 = high_codes(y);
#pragma unroll
                    for (int n = 0; n < kCols; ++n) dev::mma_f16(acc[n][2 * t + m], a0, a1, a2, a3, lo[n][j], hi[n][j]);
                }
            }
        }
        load_values();
    }

    float* mine = reinterpret_cast<float*>(sums + w * S::kSums);
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) weight[n][i] += __shfl_xor_sync(0xFFFFFFFFu, weight[n][i], d);
            const int row = 8 * n + 2 * c + i;
            if (g == 0) warp_stats[w * kRows + row] = make_float2(top[n][i], weight[n][i]);
#pragma unroll
            for (int j = 0; j < 4 * kChunks; ++j) {
                mine[row * kDim + 16 * j + g] = acc[n][j][i];
                mine[row * kDim + 16 * j + 8 + g] = acc[n][j][2 + i];
            }
        }
    }
}

// A CTA's sums of four neighbouring dimensions of a row, from its warps'; (maximum, weight) in `stat`.
template <int kChunks, int kCols>
__device__ __forceinline__ float4 join_warps(const unsigned char* sums, const float2* warp_stats, int row, int d, float2& stat) {
    using S = Shape<kChunks, kCols>;
    float m = kLowest, wt = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) m = fmaxf(m, warp_stats[i * S::kRows + row].x);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        const float2 st = warp_stats[i * S::kRows + row];
        const float f = exp2_of(st.x - m);
        const float4 v = *reinterpret_cast<const float4*>(sums + i * S::kSums + (row * S::kDim + d) * 4);
        wt += st.y * f;
        sum.x += v.x * f, sum.y += v.y * f, sum.z += v.z * f, sum.w += v.w * f;
    }
    stat = make_float2(m, wt);
    return sum;
}

template <int kChunks, int kCols>
__global__ void __launch_bounds__(kThreads, Shape<kChunks, kCols>::kCtasOfSm) kv8_attn_kernel(const AttnParams p) {
    using S = Shape<kChunks, kCols>;
    constexpr int kDim = S::kDim, kRows = S::kRows;
    extern __shared__ float4 shared[];
    unsigned char* sums = reinterpret_cast<unsigned char*>(shared);                     // [warp][kRows][kDim]
    float2* warp_stats = reinterpret_cast<float2*>(sums + kWarps * S::kSums);           // [warp][kRows]
    int* warp_sums = reinterpret_cast<int*>(warp_stats + kWarps * kRows);
    int* first = warp_sums + kWarps;
    dev::programmatic_start();
    scan_line<kThreads, kUnitCells, kRows>(p, first, warp_sums);
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        const Request rq = request_of(p, b);
        if (rq.cells == 0) store_nothing(p, rq, kDim, kThreads);
        if (p.by_triple) {                                      // triples that do not exist
            const int blocks = rq.cells > 0 ? (rq.n * p.group + kRows - 1) / kRows : 0;
            for (int i = threadIdx.x; i < p.heads * p.most_blocks; i += kThreads)
                if (i % p.most_blocks >= blocks) p.open[b * p.heads * p.most_blocks + i].x = -1;
        }
    }
    if (!p.by_triple && threadIdx.x == 0) p.open[blockIdx.x].x = -1;
    const int total = first[p.B], ctas = min(static_cast<int>(gridDim.x), total);       // so that no CTA between two others has nothing
    if (static_cast<int>(blockIdx.x) >= ctas) return;
    const int begin = run_start(total, ctas, blockIdx.x), stop = run_start(total, ctas, blockIdx.x + 1);
    int pieces = 0;
    for (int u = begin; u < stop;) {
        const int b = request_at(first, p.B, u);
        const Request rq = request_of(p, b);
        const int units = (rq.cells + kUnitCells - 1) / kUnitCells, length = triple_length(units), triple = (u - first[b]) / length, at = (u - first[b]) % length;
        const int start = u - at;                               // of the triple
        const int off = max(0, at - kStart), count = max(0, min(length, stop - start) - kStart) - off;
        u = min(start + length, stop);
        if (count <= 0) continue;                               // the run ends before the triple's first unit
        const int blocks = (rq.n * p.group + kRows - 1) / kRows, h = triple / blocks, block = triple % blocks, row0 = block * kRows, rows = min(kRows, rq.n * p.group - row0);
        attend<kChunks, kCols>(p, rq, b, h, row0, off * kUnitCells, min(rq.cells, (off + count) * kUnitCells), sums, warp_stats);
        __syncthreads();
        const bool all = count == units;
        const int slot = 2 * blockIdx.x + (pieces > 0 ? 1 : 0); // what is not whole is the first piece of a run or the last
        ++pieces;
        for (int e = threadIdx.x; e < rows * kDim / 4; e += kThreads) {       // four neighbours to a thread
            const int row = e / (kDim / 4), d = e % (kDim / 4) * 4;
            float2 stat;
            const float4 sum = join_warps<kChunks, kCols>(sums, warp_stats, row, d, stat);
            if (all) {
                store_result(p, rq.n0 + (row0 + row) / p.group, static_cast<int64_t>(h * p.group + (row0 + row) % p.group) * kDim + d, sum, stat.y);
            } else {
                *reinterpret_cast<float4*>(p.sums + (static_cast<int64_t>(slot) * kRows + row) * kDim + d) = sum;
                if (d == 0) p.stats[slot * kRows + row] = stat;
            }
        }
        if (threadIdx.x == 0 && off == 0 && (p.by_triple || !all))        // the CTAs with the rest follow this one
            p.open[p.by_triple ? (b * p.heads + h) * p.most_blocks + block : blockIdx.x] =
                make_int4(all ? -1 : b, h * p.most_blocks + block, slot, static_cast<int>(((static_cast<int64_t>(start) + length) * ctas - 1) / total));
        __syncthreads();
    }
}

// The form for few triples of few keys: a cluster of CTAs to a triple, an eighth of its keys each, whose sums meet through
// distributed shared memory.  No scratch memory, no second kernel.
constexpr int kCluster = 8;

template <int kChunks, int kCols>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, Shape<kChunks, kCols>::kCtasOfSm) kv8_attn_cluster_kernel(const AttnParams p) {
    using S = Shape<kChunks, kCols>;
    constexpr int kDim = S::kDim, kRows = S::kRows, kCells = S::kCells;
    extern __shared__ float4 shared[];
    unsigned char* sums = reinterpret_cast<unsigned char*>(shared);
    float2* warp_stats = reinterpret_cast<float2*>(sums + kWarps * S::kSums);
    float2* stats = warp_stats + kWarps * kRows;                // [kRows], read by the whole cluster, as the first warp's sums are
    dev::programmatic_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int cta = blockIdx.x % kCluster, place = blockIdx.x / kCluster, triples = p.heads * p.most_blocks, b = place / triples;
    const int h = place % triples / p.most_blocks, row0 = place % p.most_blocks * kRows;
    const Request rq = request_of(p, b);
    const int rows = min(kRows, rq.n * p.group - row0);
    if (rows <= 0) return;                                      // the whole cluster
    const int steps = (rq.cells + kCells - 1) / kCells;
    attend<kChunks, kCols>(p, rq, b, h, row0, kCells * (steps * cta / kCluster), min(rq.cells, kCells * (steps * (cta + 1) / kCluster)), sums, warp_stats);
    __syncthreads();
    for (int e = threadIdx.x; e < rows * kDim / 4; e += kThreads) {
        const int row = e / (kDim / 4), d = e % (kDim / 4) * 4;
        float2 stat;
        const float4 sum = join_warps<kChunks, kCols>(sums, warp_stats, row, d, stat);
        *reinterpret_cast<float4*>(sums + (row * kDim + d) * 4) = sum;       // nobody else reads or writes the first warp's there
        if (d == 0) stats[row] = stat;
    }
    cluster.sync();
    static_assert(kRows * kDim / 4 <= kCluster * kThreads, "a thread of the cluster for every four results");
    const int e = cta * kThreads + threadIdx.x;
    if (e < rows * kDim / 4) {
        const int row = e / (kDim / 4), d = e % (kDim / 4) * 4;
        float m = kLowest, wt = 0.0f;
        float2 st[kCluster];
        float4 v[kCluster], sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {
            st[i] = cluster.map_shared_rank(stats, i)[row];
            v[i] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(sums, i) + (row * kDim + d) * 4);
            m = fmaxf(m, st[i].x);
        }
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {
            const float f = exp2_of(st[i].x - m);
            wt += st[i].y * f;
            sum.x += v[i].x * f, sum.y += v[i].y * f, sum.z += v[i].z * f, sum.w += v[i].w * f;
        }
        store_result(p, rq.n0 + (row0 + row) / p.group, static_cast<int64_t>(h * p.group + (row0 + row) % p.group) * kDim + d, sum, wt);
    }
    cluster.sync();                                             // nobody reads this CTA's sums any more
}

template <int kChunks, int kCols>
constexpr size_t base_bytes() { return kWarps * Shape<kChunks, kCols>::kSums + (kWarps + 1) * 8 * kCols * sizeof(float2); }
template <int kChunks, int kCols>
size_t line_bytes(int B) { return base_bytes<kChunks, kCols>() + (kWarps + B + 1) * sizeof(int); }

// Up to here a cluster to a triple, where all of them fit the GPU at once.  What decides is the longest that the table or the window
// allows: a request's own length is only known on the device.  As a line or as clusters, us, 8 query heads to a key head: 8 triples of heads of 128 18.8 / 14.3 at 4000
// keys, 20.8 / 20.5 at 8000, 22.8 / 30.7 at 16000; 32 triples 29.0 / 24.6 at 8000, 59.7 / 59.4 at 32000; 8 of 64 16.7 / 14.3 and 16.8 / 18.4, 4 of 256 20.8 / 20.5 and
// 22.8 / 30.7 at 4000 and 8000.
constexpr int kClusterKeys = 8192;

template <int kChunks, int kCols>
spdp_status launch_form(AttnParams p, int device, int sms, cudaStream_t s) {
    constexpr int kDim = 64 * kChunks, kRows = 8 * kCols;
    static std::mutex mu;
    static int resident[64] = {};                               // CTAs of an SM
    int per_sm;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (resident[device] == 0) {
            SPDP_CUDA_TRY(cudaFuncSetAttribute(kv8_attn_kernel<kChunks, kCols>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(line_bytes<kChunks, kCols>(kMostRequests))));
            SPDP_CUDA_TRY(cudaFuncSetAttribute(kv8_attn_cluster_kernel<kChunks, kCols>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(base_bytes<kChunks, kCols>())));
            SPDP_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident[device], kv8_attn_kernel<kChunks, kCols>, kThreads, line_bytes<kChunks, kCols>(64)));
        }
        per_sm = resident[device] > 0 ? resident[device] : 1;
    }
    const int most_rows = p.first == nullptr ? p.group : p.N * p.group < p.most_rows ? p.N * p.group : p.most_rows;
    p.most_blocks = (most_rows + kRows - 1) / kRows;
    const int triples = p.heads * p.most_blocks;
    const int64_t cells = p.window > 0 ? p.window / kCell + (p.first == nullptr ? 1 : p.N) / kCell + p.sinks / kCell + 3 : p.most_cells;
    const int longest = static_cast<int>(cells < p.most_cells ? cells : p.most_cells);
    if (static_cast<int64_t>(longest) * kCell <= kClusterKeys && static_cast<int64_t>(p.B) * triples * kCluster <= static_cast<int64_t>(per_sm) * sms) {
        SPDP_CUDA_TRY(launch_programmatic(kv8_attn_cluster_kernel<kChunks, kCols>, dim3(static_cast<unsigned>(p.B * triples * kCluster)), kThreads, base_bytes<kChunks, kCols>(), s, p));
        return SPDP_OK;
    }
    // no more CTAs than there can be units
    const int64_t most = static_cast<int64_t>(p.B) * ((p.most_cells + kUnitCells - 1) / kUnitCells) * triples;
    const int ctas = static_cast<int>(most < static_cast<int64_t>(per_sm) * sms ? most : per_sm * sms);
    const size_t sums = 2ull * ctas * kRows * kDim * sizeof(float), stats = 2ull * ctas * kRows * sizeof(float2);
    void* scratch = nullptr;
    const spdp_status st = scratch_alloc(device, sums + stats + ctas * sizeof(int4), s, &scratch);
    if (st != SPDP_OK) return st;
    p.sums = static_cast<float*>(scratch);
    p.stats = reinterpret_cast<float2*>(static_cast<char*>(scratch) + sums);
    p.by_triple = static_cast<int64_t>(p.B) * triples <= ctas;
    const int places = p.by_triple ? p.B * triples : ctas;
    p.open = reinterpret_cast<int4*>(static_cast<char*>(scratch) + sums + stats);
    cudaError_t e = launch_programmatic(kv8_attn_kernel<kChunks, kCols>, dim3(static_cast<unsigned>(ctas)), kThreads, line_bytes<kChunks, kCols>(p.B), s, p);
    if (e == cudaSuccess)
        e = launch_programmatic(ctas >= kJoinFew * places ? attn_join_few_kernel<kDim, kRows> : attn_join_kernel<kDim, kRows>, dim3(static_cast<unsigned>(places), static_cast<unsigned>(most_rows < kRows ? most_rows : kRows)), kJoinThreads, 0, s, p);
    const cudaError_t freed = cudaFreeAsync(scratch, s);
    SPDP_CUDA_TRY(e);
    SPDP_CUDA_TRY(freed);
    return SPDP_OK;
}

template <int kChunks>
spdp_status launch_dim(const AttnParams& p, int device, int sms, cudaStream_t s) {
    if constexpr (kChunks < 4) {                                // heads of 256 leave no registers for 16 columns
        // Rows of a request, on average, that make two blocks of columns worth their place; beside prompts, whose tokens the number N has too, those
        // of one token.  One or two, us, 8 key heads of 128: 48 requests behind 4000 keys 98 / 120 at 8 rows, 157 / 124 at 16, 218 / 202 at 24, 497 / 360 at 64;
        // one behind 65536 43 / 50, 64 / 50, 68 / 76, 172 / 125; one behind 2000 12 / 14, 12 / 16, 13 / 16, 21 / 16.
        if (p.most_rows < INT32_MAX ? p.group > 8 : static_cast<int64_t>(p.N) * p.group > 8ll * p.B) return launch_form<kChunks, 2>(p, device, sms, s);
    }
    return launch_form<kChunks, 1>(p, device, sms, s);
}

int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

}  // namespace

spdp_status launch_kv8_store(const Kv8StoreCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    StoreParams p = {};
    p.k = call.k, p.v = call.v, p.table = call.table, p.first = call.first, p.length = call.length, p.cache = call.cache, p.k_values = call.k_values, p.v_values = call.v_values;
    p.ldk = call.ldk, p.ldv = call.ldv, p.ldk_values = call.ldk_values, p.ldv_values = call.ldv_values, p.table_stride = call.table_stride;
    p.pages = static_cast<unsigned>(call.pages), p.N = static_cast<int>(call.N), p.B = static_cast<int>(call.B), p.heads = call.kv_heads;
    p.cells_shift = log2_of(call.page_tokens / kCell), p.most_cells = static_cast<int>(call.table_pages) << p.cells_shift;
    const bool f32 = call.vdt == SPDP_Y_F32;
    auto fours = [](const void* x, int64_t ld, int64_t size) { return rows_alignment(x, ld, size) >= 4 * size; };
    const bool wide = fours(p.k, p.ldk, 2) && fours(p.v, p.ldv, f32 ? 4 : 2) && fours(p.k_values, p.ldk_values, 2) && fours(p.v_values, p.ldv_values, 2);
    switch (call.head_dim) {
        case 64: SPDP_CUDA_TRY(f32 ? (launch_store<float, 64>(p, wide, sms, s)) : (launch_store<__half, 64>(p, wide, sms, s))); break;
        case 128: SPDP_CUDA_TRY(f32 ? (launch_store<float, 128>(p, wide, sms, s)) : (launch_store<__half, 128>(p, wide, sms, s))); break;
        default: SPDP_CUDA_TRY(f32 ? (launch_store<float, 256>(p, wide, sms, s)) : (launch_store<__half, 256>(p, wide, sms, s)));
    }
    return SPDP_OK;
}

spdp_status launch_attn_kv8(const Kv8AttnCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    AttnParams p = {};
    p.q = call.q, p.cache = call.cache, p.table = call.table, p.first = call.first, p.length = call.length, p.y = call.y, p.mask = call.mask;
    p.ldq = call.ldq, p.ldy = call.ldy, p.table_stride = call.table_stride, p.mask_stride = call.mask_stride, p.pages = static_cast<unsigned>(call.pages);
    p.N = static_cast<int>(call.N), p.B = static_cast<int>(call.B), p.heads = call.kv_heads, p.group = call.q_heads / call.kv_heads;
    p.cells_shift = log2_of(call.page_tokens / kCell), p.most_cells = static_cast<int>(call.table_pages) << p.cells_shift;
    p.low_rows = 0, p.most_rows = INT32_MAX;
    const int64_t keys = static_cast<int64_t>(p.most_cells) * kCell;
    p.window = call.window < keys ? static_cast<int>(call.window) : 0;         // a window of all keys is none
    p.sinks = static_cast<int>(call.sinks < keys ? call.sinks : keys);
    constexpr float kLog2e = 1.4426950408889634f;
    p.scale = call.scale * kLog2e;
    p.cap = call.cap * kLog2e;
    p.cap_inv = call.cap > 0.0f ? fminf(1.0f / p.cap, FLT_MAX) : 0.0f;         // never Inf, for a score may be 0
    p.cap_near = 0.25f * p.cap;
    p.thr = call.thr;
    p.wide_q = rows_aligned16(p.q, p.ldq, 2), p.wide_y = rows_alignment(p.y, p.ldy, 2) >= 8;
    // requests of more rows than kFewRows are the other kernel's; where no request can have as few, or as many, one of the two is not launched
    const int64_t rows = static_cast<int64_t>(p.N) * p.group;
    const bool prompts = p.first != nullptr && rows > kFewRows;
    if (prompts) p.most_rows = kFewRows;
    if (!prompts || p.B > 1) {
        const spdp_status few = call.head_dim == 64 ? launch_dim<1>(p, device, sms, s) : call.head_dim == 128 ? launch_dim<2>(p, device, sms, s) : launch_dim<4>(p, device, sms, s);
        if (few != SPDP_OK || !prompts) return few;
    }
    p.low_rows = p.B > 1 ? kFewRows + 1 : 0, p.most_rows = INT32_MAX;
    return launch_kv8_prompt(p, call.head_dim, device, sms, s);
}

}  // namespace spdp
