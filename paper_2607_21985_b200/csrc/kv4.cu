// A paged key/value cache of 4-bit codes: storing rows (what a q/k/v projection and the rotation left), and the attention of
// one new token per request over it, whose output is the input of a dynamically pruned o-projection and comes with its keep
// mask, as spdp_swiglu_dp's does.
//
// Layout of the cache (spdp.h): per page and key head the codes of the keys [P][D/2], of the values [P][D/2], the scales of the keys
// [P][D/32] and of the values [P][D/32].  In a row of codes the dimension 32 g + 8 c + j is nibble j of word c D/32 + g: so the
// four lanes that share a key in a matrix product's fragment each read one run of 16 bytes (D = 128), and what a lane holds
// for one step of the product all belongs to one scale.
#include <cooperative_groups.h>

#include <cfloat>
#include <mutex>

#include "mma_f16.cuh"
#include "spdp_internal.h"

namespace cg = cooperative_groups;

namespace spdp {
namespace {

// ---- storing ----------------------------------------------------------------------------------------------------------------

constexpr int kStoreThreads = 256;

struct StoreParams {
    const __half* k;
    const void* v;
    const int64_t* slot;
    unsigned char* cache;
    __half* k_values;
    __half* v_values;
    int64_t ldk, ldv, ldk_values, ldv_values, N, pages;
    int heads, dim, page_shift, row_shift;      // pieces of 8 dimensions in a row: 2^row_shift
};

// x / s, correctly rounded where the quotient is a number of 24 bits (as where a code lies half way between two, which are n +
// 1/2) and else to within a step: a product with the reciprocal (to within a step itself), corrected by its exact remainder
// (Markstein).  Quotients of fp16 numbers that are not half way are 2^-12 and more of their size away from it, and sevenths 2^-15
// and more away from the middle of two fp16 numbers, so rounding gives what it gives for the true quotient.
__device__ __forceinline__ float quotient(float x, float s, float reciprocal) {
    const float q = x * reciprocal;
    return fmaf(fmaf(-q, s, x), reciprocal, q);
}

// A thread takes 8 dimensions (a piece; four neighbouring threads a scale) of kTokens tokens, whose loads are on their way at
// once.  blockDim.x: the pieces of a token, or 256 of them at a time; blockDim.y: tokens.  kWide: 16-byte accesses.
// 16384 tokens of 8 heads of 128, 32-bit values, both written back as fp16: 33.6 us, 187 MB at 5.6 TB/s.
template <typename T, bool kWide, int kTokens>
__device__ __forceinline__ void store_rows(const StoreParams& p, const T* from, int64_t ld, __half* values, int64_t ld_values, bool is_v) {
    const int P = 1 << p.page_shift, groups = p.dim / 32, row_bytes = p.dim / 2;
    const unsigned head_bytes = P * (p.dim + p.dim / 8), page_bytes = p.heads * head_bytes;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * (kTokens * blockDim.y) + threadIdx.y;
    const unsigned four = 0xFu << ((threadIdx.y * blockDim.x + threadIdx.x) & 28);      // the lanes of a scale come and go together
    for (int t = threadIdx.x; t < p.heads << p.row_shift; t += blockDim.x) {
        float x[kTokens][8];
        int64_t slot[kTokens];
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            const int64_t n = n0 + j * blockDim.y;
            if (n >= p.N) continue;
            slot[j] = p.slot[n];
            dev::load_floats<T, kWide>(from + n * ld + 8 * t, x[j]);
        }
        const int piece = t & ((1 << p.row_shift) - 1), c = piece & 3, g = piece >> 2;
        unsigned char* head = p.cache + (t >> p.row_shift) * static_cast<int64_t>(head_bytes);
        unsigned char* word_at = head + (is_v ? P * row_bytes : 0) + 4 * (c * groups + g);
        unsigned char* scale_at = head + 2 * P * row_bytes + (is_v ? P * groups * 2 : 0) + 2 * g;
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            const int64_t n = n0 + j * blockDim.y;
            if (n >= p.N) continue;
            if constexpr (sizeof(T) == 4) {                      // 32-bit rows count as the fp16 row they round to
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float2 f = __half22float2(__floats2half2_rn(x[j][e], x[j][e + 1]));
                    x[j][e] = f.x, x[j][e + 1] = f.y;
                }
            }
            float top = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[j][e]));
            top = fmaxf(top, __shfl_xor_sync(four, top, 1));
            top = fmaxf(top, __shfl_xor_sync(four, top, 2));
            const __half scale = __float2half_rn(quotient(top, 7.0f, 1.0f / 7.0f));
            const float s = __half2float(scale);
            float reciprocal;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(reciprocal) : "f"(s));
            if (!(s > 0.0f)) reciprocal = 0.0f;
            // Adding 1.5 2^23 + 8 rounds to a whole number, ties to even, and leaves it, 8 more, in the lowest bits
            constexpr float kWhole = 12582912.0f + 8.0f;
            constexpr uint32_t kWholeBits = 0x4B400000u;
            float q[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) q[e] = quotient(x[j][e], s, reciprocal);
            if (!(s >= 0x1p-14f && s < 0x1p15f)) {               // else 7 (1 + 2^-11) at most; a subnormal scale may be far off a seventh
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = fminf(fmaxf(q[e], -7.0f), 7.0f);
            }
            uint32_t word = 0, offset = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float whole = q[e] + kWhole;
                word += __float_as_uint(whole) << (4 * e);
                offset += kWholeBits << (4 * e);
                x[j][e] = (whole - kWhole) * s;
            }
            word -= offset;
            const int64_t page = slot[j] >> p.page_shift;
            if (slot[j] >= 0 && page < p.pages) {
                const uint64_t first = static_cast<uint64_t>(static_cast<unsigned>(page)) * page_bytes;
                const unsigned at = static_cast<unsigned>(slot[j]) & (P - 1);
                *reinterpret_cast<uint32_t*>(word_at + first + at * row_bytes) = word;
                if (c == 0) *reinterpret_cast<__half*>(scale_at + first + at * groups * 2) = scale;
            }
            if (values != nullptr) dev::store_halves<kWide>(values + n * ld_values + 8 * t, x[j]);
        }
    }
}

template <typename V, bool kWide, int kTokens>
__global__ void __launch_bounds__(kStoreThreads) kv4_store_kernel(const StoreParams p) {
    dev::programmatic_start();
    if (blockIdx.y == 0) store_rows<__half, kWide, kTokens>(p, p.k, p.ldk, p.k_values, p.ldk_values, false);
    else store_rows<V, kWide, kTokens>(p, static_cast<const V*>(p.v), p.ldv, p.v_values, p.ldv_values, true);
}

template <typename V, bool kWide>
cudaError_t launch_store(const StoreParams& p, int sms, cudaStream_t s) {
    const int pieces = p.heads << p.row_shift;
    const dim3 block(pieces < kStoreThreads ? pieces : kStoreThreads, pieces < kStoreThreads ? kStoreThreads / pieces : 1);
    // two tokens to a thread where that still fills the GPU
    const int64_t ctas = (p.N + block.y - 1) / block.y;
    if (ctas > 8 * sms) return launch_programmatic(kv4_store_kernel<V, kWide, 2>, dim3(static_cast<unsigned>((ctas + 1) / 2), 2), block, 0, s, p);
    return launch_programmatic(kv4_store_kernel<V, kWide, 1>, dim3(static_cast<unsigned>(ctas), 2), block, 0, s, p);
}

// ---- attention --------------------------------------------------------------------------------------------------------------
//
// The keys of all (request, key head, block of query heads) triples, 64 to a unit, stand in one line that is cut into equal runs,
// one to a CTA: so one long request and many short ones alike occupy the whole GPU, whatever the lengths are, which only
// the device knows.  A run that holds a triple's every key writes its output; else CTAs leave a partial sum of it, with its
// maximum and its weight, and a second kernel joins them in the order of the keys.
//
// Inside a CTA each warp takes 32 keys at a time, copied to shared memory one step ahead.  Scores are K q^T and outputs V^T P^T on
// mma.sync, with the query heads of the key head as the 8 columns (so that up to 8 heads cost no more than one, and 16 share
// what was decoded).  A key's code n goes into the products as it is: masked out of its word, four bits are a subnormal fp16
// number, n 2^-24 or n 2^-20, which the products take exactly; that it stands for n - 8 is one more product, of the scales.  So a
// pair of codes costs one logical operation.  The keys' scales multiply the 32-bit sums of their 32 dimensions.  The values'
// codes become exact fp16 numbers n - 8, and their scales multiply the softmax's weights, once for the 32 dimensions of a scale,
// before these are rounded to fp16 (2^-11): the one rounding besides the result's.
// What bounds it: the chains of a warp's instructions at the 16 warps that the registers allow (issued: 0.64 a cycle and scheduler, half
// of them on the integer pipe, the tensor pipe 23 % busy).  48 requests of up to 16384 keys, 64 and 8 heads of 128: 107 us for 421 MB
// (3.9 TB/s), 740 instructions to a warp's 32 keys.  Five CTAs to an SM spill (153 us), three take as long as four.

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kUnit = 64;               // keys
constexpr int kMostRequests = 4096;
constexpr float kLowest = -1.0e30f;     // stands for "no score yet"
constexpr float kHeadroom = 12.0f;      // weights are at most 2^(kHeadroom + kSlack), 2^kSlack where the scales are as large as they can be (2^14):
constexpr float kSlack = 1.5f;          // their products with the scales are below 2^15.5

struct AttnParams {
    const __half* q;
    const unsigned char* cache;
    const int32_t* table;
    const int32_t* length;
    __half* y;
    uint32_t* mask;
    float* sums;                        // [2 CTAs][rows][dim]
    float2* stats;                      // [2 CTAs][rows]: maximum, weight
    int4* open;                         // triples that several CTAs have: request (-1: none), triple, slot of the first sum, last CTA
    bool by_triple;                     // a place of `open` for each triple; else for each CTA, of the triple that begins there
    int64_t ldq, ldy, table_stride, table_pages, mask_stride;
    unsigned pages;
    int B, heads, group, row_blocks, page_shift;
    float scale, cap, cap_inv, cap_near;        // scores in powers of two; 1 / cap, and a quarter of the cap
    bool wide_q, wide_y;
    int64_t window;
    float thr;
};

struct Span {
    int low, end, units;                // keys of the request: low .. end - 1 (low a multiple of 16), in units
};
__device__ __forceinline__ Span span_of(const AttnParams& p, int b) {
    const int64_t most = p.table_pages << p.page_shift;
    const int64_t n = p.length[b] < 0 ? 0 : p.length[b] < most ? p.length[b] : most;
    Span s;
    s.end = static_cast<int>(n);
    s.low = p.window > 0 && n > p.window ? static_cast<int>(n - p.window) & ~15 : 0;
    s.units = (s.end - s.low + kUnit - 1) / kUnit;
    return s;
}

// A triple costs what its units do and, for its query heads and its sums, as much as kStart more: it is that long in the line
// that is cut into runs.  (Us with 0, 3 and 6, 64 and 8 heads: 48 requests of 1 to 16384 keys 153, 143, 134; 256 of 1 to 1024 131, 85, 79; 128
// with heads of 64, lengths to 4096 even in their logarithm, 77, 48, 44; 16 of up to 8192 50, 42, 42.)
constexpr int kStart = 6;               // spdp_attn_kv4 counts on 7 at most when it checks that a line's length fits 32 bits
__device__ __forceinline__ int triple_length(int units) { return units > 0 ? units + kStart : 0; }

// Where the run of CTA i begins, of `ctas` that share a line of `total`.
__device__ __forceinline__ int run_start(int total, int ctas, int i) { return static_cast<int>(static_cast<int64_t>(total) * i / ctas); }

// Where in the line every request begins, into shared memory (all threads; ends with a barrier).
__device__ void scan_units(const AttnParams& p, int* first, int* warp_sums) {
    const int each = (p.B + kThreads - 1) / kThreads, b0 = threadIdx.x * each, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int mine = 0;
    for (int b = b0; b < b0 + each && b < p.B; ++b) mine += triple_length(span_of(p, b).units) * p.heads * p.row_blocks;
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
        first[b] = at;
        at += triple_length(span_of(p, b).units) * p.heads * p.row_blocks;
    }
    if (b0 < p.B && b0 + each >= p.B) first[p.B] = at;
    __syncthreads();
}

// (w & mask) | bits as one operation (with two constants in the instruction the compiler makes two of it).
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
    return r;
}
__device__ __forceinline__ uint32_t low_pair(uint32_t w) {       // nibbles 0 and 4 of w, as fp16 numbers minus 8
    const uint32_t v = and_or(w, 0x000F000Fu, 0x64006400u);      // 1024 + n
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&v), __half2half2(__ushort_as_half(0x6408)));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t high_pair(uint32_t w) {      // nibbles 1 and 5
    const uint32_t v = and_or(w, 0x00F000F0u, 0x54005400u);      // 64 + n
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&v), __half2half2(__ushort_as_half(0x5480)));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// pair i: nibbles i and i + 4
__device__ __forceinline__ void pairs_of(uint32_t w, uint32_t (&out)[4]) {
    out[0] = low_pair(w), out[1] = high_pair(w), out[2] = low_pair(w >> 8), out[3] = high_pair(w >> 8);
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// cap * tanh(s / cap): up to a quarter of the cap by the series of tanh, which is off by 2^-21 of s (most of it where it is cut off)
// however large the cap is; beyond, as 1 - 2 / (e^2x + 1), which keeps its limits and is off by 2^-21 of the cap, 2^-19 of s.
// 48 requests of up to 16384 keys: 116 us without a cap, 122 where a lane's scores stay below a quarter of it, 138 where they often do not.
__device__ __forceinline__ float capped_near(const AttnParams& p, float s) {
    const float x = s * p.cap_inv, t = x * x;
    return fmaf(s * t, fmaf(fmaf(-17.0f / 315.0f, t, 2.0f / 15.0f), t, -1.0f / 3.0f), s);
}
__device__ __forceinline__ float capped_far(const AttnParams& p, float s) {
    constexpr float kTwoLog2e = 2.8853900817779268f;
    return p.cap * (1.0f - __fdividef(2.0f, exp2_of(s * p.cap_inv * kTwoLog2e) + 1.0f));
}

// kWords 32-bit words (1, 2, 4 or 8) from an address that is a multiple of their size (16 at most).
template <int kWords>
__device__ __forceinline__ void load_words(const unsigned char* at, uint32_t (&w)[kWords]) {
    if constexpr (kWords == 1) w[0] = *reinterpret_cast<const uint32_t*>(at);
    else if constexpr (kWords == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(at);
        w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(at)[i];
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
    }
}

// 16 keys in shared memory, as a warp's asynchronous copies leave them: four runs of the page's head.  The values' rows are 16
// bytes further apart than in the page, so that a lane's reads of rows 2 c meet other banks than its neighbours'.
template <int kGroups>
struct Chunk {
    static constexpr int kRow = 16 * kGroups, kValueRow = kRow + 16;
    static constexpr int kValues = 16 * kRow, kKeyScales = kValues + 16 * kValueRow, kValueScales = kKeyScales + 32 * kGroups;
    static constexpr int kBytes = kValueScales + 32 * kGroups;
};
constexpr int kStages = 2;              // of a warp, two chunks each: one is read while the other is on its way

__device__ __forceinline__ void copy16(uint32_t to, const unsigned char* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy16_if(bool on, uint32_t to, const unsigned char* from) {
    asm volatile("{\n .reg .pred p;\n setp.ne.s32 p, %2, 0;\n @p cp.async.cg.shared.global [%0], [%1], 16;\n}" ::"r"(to), "l"(from), "r"(static_cast<int>(on)) : "memory");
}

// 16 keys into a chunk.  The lane's addresses: `to`, `keys` of its 16 bytes of the first 512 of their codes and `scale` of its 16
// bytes of the scales (keys' and values': 4 kGroups lanes have some); `values`: how far behind the keys' codes the values' are;
// value_to, scale_to: the lane's places for these, from `to`.
template <int kGroups>
__device__ __forceinline__ void copy_chunk(uint32_t to, const unsigned char* keys, const unsigned char* scale, int values, int value_to, int scale_to, bool has_scale) {
    using C = Chunk<kGroups>;
    constexpr int kRows = 32 / kGroups;             // of 512 bytes
#pragma unroll
    for (int i = 0; i < 512 * kGroups / 1024; ++i) {
        copy16(to + 512 * i, keys + 512 * i);
        copy16(to + value_to + kRows * C::kValueRow * i, keys + values + 512 * i);
    }
    copy16_if(has_scale, to + scale_to, scale);
}

// Four columns of a request's output and their bits of its mask; 8 neighbouring lanes have the columns of a word.
__device__ __forceinline__ void store_result(const AttnParams& p, int b, int64_t column, float4 sum, float weight) {
    const float f[4] = {sum.x, sum.y, sum.z, sum.w};
    __half y[4];
    unsigned keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = __float2half_rn(weight > 0.0f || weight != weight ? f[i] / weight : 0.0f);
        keep |= (fabsf(__half2float(y[i])) <= p.thr ? 0u : 1u) << i;
    }
    __half* to = p.y + b * p.ldy + column;
    if (p.wide_y) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(y);
    else to[0] = y[0], to[1] = y[1], to[2] = y[2], to[3] = y[3];
    keep <<= 4 * (threadIdx.x & 7);
    const unsigned mine = 0xFFu << (threadIdx.x & 24);          // the lanes of a word come together
#pragma unroll
    for (int d = 1; d < 8; d *= 2) keep |= __shfl_xor_sync(mine, keep, d);
    if (p.mask != nullptr && (threadIdx.x & 7) == 0) p.mask[b * p.mask_stride + column / 32] = keep;
}

// A CTA's warps over the keys k0 .. k1 - 1 of a triple: a warp's sums [kRows][kDim] end up in its part of `rings`, its maxima and
// weights in warp_stats [warp][kRows].  kGroups = D / 32; kCols: blocks of 8 query heads.
template <int kGroups, int kCols>
struct Shape {
    static constexpr int kDim = 32 * kGroups, kRows = 8 * kCols;
    static constexpr int kRing = 2 * kStages * Chunk<kGroups>::kBytes;      // bytes of a warp
    static constexpr int kCtasOfSm = kGroups == 8 ? 2 : kCols == 2 ? 3 : 4; // that the registers are cut for
    static_assert(kRing >= kRows * kDim * 4 && kRing % 16 == 0, "a warp's sums take the place of its chunks");
};

template <int kGroups, int kCols>
__device__ __forceinline__ void attend(const AttnParams& p, int b, int h, int row0, int k0, int k1, int end, unsigned char* rings, float2* warp_stats) {
    using S = Shape<kGroups, kCols>;
    constexpr int kDim = S::kDim, kRows = S::kRows, kRing = S::kRing;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int P = 1 << p.page_shift, rows = min(kRows, p.group - row0);
    const unsigned head_bytes = P * 36 * kGroups, page_bytes = head_bytes * p.heads;
    const int window_low = p.window > 0 && end > p.window ? static_cast<int>(end - p.window) : 0;
    const int32_t* table = p.table + b * p.table_stride;

    // the warp's stages: every fourth one of the run.  Each lane knows the page of a chunk of 16 of them, and of the next 16
    using C = Chunk<kGroups>;
    const int stages = ((k1 - k0 + 31) / 32 - w + kWarps - 1) / kWarps;
    int key = k0 + 32 * w, asked = key;                         // the first key of the stage that is worked on, and that is asked for
    auto page_of = [&](int i) {                                 // of the stages i .. i + 15
        const int at = k0 + 32 * (w + kWarps * (i + (lane >> 1))) + 16 * (lane & 1);
        return at < k1 ? table[at >> p.page_shift] : -1;
    };
    int pages = page_of(0), pages_after = page_of(16);
    unsigned there = 0;                                         // two bits for each stage that was asked for: which of its chunks exist
    const unsigned char* codes = p.cache + h * static_cast<int64_t>(head_bytes) + 16 * lane;
    const unsigned char* scales = codes + 2 * P * C::kRow + (lane < 2 * kGroups ? 0 : P * 2 * kGroups - 32 * kGroups);
    const int values = P * C::kRow, value_to = C::kValues + lane / kGroups * C::kValueRow + lane % kGroups * 16 - 16 * lane, scale_to = C::kKeyScales;
    uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(rings)) + w * kRing + 16 * lane;
    uint32_t flip = 2 * C::kBytes;                              // to the other stage, and back
    auto ask = [&](int i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const unsigned page = __shfl_sync(0xFFFFFFFFu, pages, 2 * i + j & 31);
            const bool ok = page < p.pages;                     // negative ones are large here; the first page stands in for what does not exist
            there = there << 1 | (ok ? 1u : 0u);
            const uint64_t first = static_cast<uint64_t>(ok ? page : 0u) * page_bytes;
            const int at = (asked + 16 * j) & (P - 1);
            copy_chunk<kGroups>(to + j * C::kBytes, codes + first + at * C::kRow, scales + first + at * 2 * kGroups, values, value_to, scale_to, lane < 4 * kGroups);
        }
        to += flip, flip = -flip, asked += 32 * kWarps;
        if ((i & 15) == 15) pages = pages_after, pages_after = page_of(i + 17);
    };
    if (stages > 0) ask(0);
    asm volatile("cp.async.commit_group;" ::: "memory");

    // The query heads as the products' columns, in the order that the codes' pairs have.  A code n is taken from its word by
    // one logical operation, as the subnormal fp16 number n 2^-24 or, four bits up, n 2^-20: the heads are scaled by a power of two
    // of their own (2^10 <= largest < 2^11, so that it costs no digits) and 2^4 more where the former meet them.  That a code
    // stands for n - 8 takes a product of its own, of the keys' scales and -8 times the sums of the heads' 32 dimensions: its
    // columns k hold the scales twice, against the upper and the lower 11 bits of these sums.
    uint32_t q[kCols][2 * kGroups][2];
    uint32_t minus[kCols][2] = {};
    float factor[kCols][2];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
        const int row = 8 * n + g;
        const __half* at = p.q + b * p.ldq + static_cast<int64_t>(h * p.group + row0 + row) * kDim + 8 * c;
        float x[kGroups][8], most = 0.0f;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            if (row >= rows) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
            } else if (p.wide_q) dev::load_floats<__half, true>(at + 32 * i, x[i]);
            else dev::load_floats<__half, false>(at + 32 * i, x[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[i][j]));
        }
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        const int exponent = max(100, min(150, __float_as_int(most) >> 23 & 255));       // of 0, Inf and NaN: a plain number
        const float up = __int_as_float((127 + 10 + 127 - exponent) << 23), down = __int_as_float((127 + 20 - 10 - 127 + exponent) << 23);
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = j & 1 ? up : 16.0f * up;
                const __half2 v = __floats2half2_rn(x[i][j] * f, x[i][j + 4] * f);
                q[n][2 * i + (j >> 1)][j & 1] = *reinterpret_cast<const uint32_t*>(&v);
            }
        }
#pragma unroll
        for (int i = 0; i < kGroups; i += 2) {              // two scales to a register: the word i / 2 of the keys' scales
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[m] += x[i + m][j];
                sum[m] += __shfl_xor_sync(0xFFFFFFFFu, sum[m], 1);
                sum[m] += __shfl_xor_sync(0xFFFFFFFFu, sum[m], 2);
                sum[m] *= -8.0f * up * 0x1p-20f;
            }
            const __half2 high = __floats2half2_rn(sum[0], sum[1]);
            const float2 h2 = __half22float2(high);
            const __half2 low = __floats2half2_rn(sum[0] - h2.x, sum[1] - h2.y);
            if (c == i / 2) minus[n][0] = *reinterpret_cast<const uint32_t*>(&high);
            if (kGroups == 8) {
                if (c == i / 2) minus[n][1] = *reinterpret_cast<const uint32_t*>(&low);
            } else if (c == i / 2 + kGroups / 2) {
                minus[n][0] = *reinterpret_cast<const uint32_t*>(&low);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) factor[n][i] = p.scale * __shfl_sync(0xFFFFFFFFu, down, 4 * (2 * c + i));
    }
    float acc[kCols][2 * kGroups][4] = {};
    float top[kCols][2], weight[kCols][2], headroom = kHeadroom;
    __half2 scale_limit = __float2half2_rn(exp2f(14.0f - kHeadroom));
#pragma unroll
    for (int n = 0; n < kCols; ++n) top[n][0] = top[n][1] = kLowest, weight[n][0] = weight[n][1] = 0.0f;

    const unsigned char* stage = rings + w * kRing;
    int other = 2 * C::kBytes;
    for (int i = 0; i < stages; ++i, key += 32 * kWarps, stage += other, other = -other) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();                                           // all lanes' copies are there, and all have read the stage before
        const unsigned have = there;
        if (i + 1 < stages) ask(i + 1);
        asm volatile("cp.async.commit_group;" ::: "memory");
        if ((have & 3) == 0) continue;                          // pages that do not exist
        const bool whole = (have & 3) == 3 && key >= window_low && key + 32 <= k1;
        auto counts = [&](int at, int j) { return at >= window_low && at < k1 && (have >> (1 - j) & 1); };

        float score[kCols][2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const unsigned char* chunk = stage + j * C::kBytes;
            uint32_t k[2][kGroups], ks[2][kGroups / 2];     // keys g and g + 8
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                load_words<kGroups>(chunk + (g + 8 * m) * C::kRow + c * 4 * kGroups, k[m]);
                load_words<kGroups / 2>(chunk + C::kKeyScales + (g + 8 * m) * 2 * kGroups, ks[m]);
            }
            uint32_t both[2];                               // the lane's part of the scales' product
#pragma unroll
            for (int m = 0; m < 2; ++m) both[m] = *reinterpret_cast<const uint32_t*>(chunk + C::kKeyScales + (g + 8 * m) * 2 * kGroups + c % (kGroups / 2) * 4);
#pragma unroll
            for (int n = 0; n < kCols; ++n)
                dev::mma_f16_from(score[n][j], 0.0f, 0.0f, 0.0f, 0.0f, both[0], both[1], kGroups == 8 ? both[0] : 0u, kGroups == 8 ? both[1] : 0u, minus[n][0], minus[n][1]);
#pragma unroll
            for (int t = 0; t < kGroups; ++t) {
                const float2 s0 = __half22float2(*reinterpret_cast<const __half2*>(&ks[0][t / 2])), s1 = __half22float2(*reinterpret_cast<const __half2*>(&ks[1][t / 2]));
                const float f0 = t & 1 ? s0.y : s0.x, f1 = t & 1 ? s1.y : s1.x;
                const uint32_t a = k[0][t], b = k[1][t], a8 = a >> 8, b8 = b >> 8;
                constexpr uint32_t kLow = 0x000F000Fu, kHigh = 0x00F000F0u;
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
                    float d[4];
                    dev::mma_f16_from(d, 0.0f, 0.0f, 0.0f, 0.0f, a & kLow, b & kLow, a & kHigh, b & kHigh, q[n][2 * t][0], q[n][2 * t][1]);
                    dev::mma_f16(d, a8 & kLow, b8 & kLow, a8 & kHigh, b8 & kHigh, q[n][2 * t + 1][0], q[n][2 * t + 1][1]);
                    score[n][j][0] += d[0] * f0, score[n][j][1] += d[1] * f0;
                    score[n][j][2] += d[2] * f1, score[n][j][3] += d[3] * f1;
                }
            }
        }
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int m = 0; m < 4; ++m) score[n][j][m] *= factor[n][m & 1];
            }
            if (p.cap > 0.0f) {
                float most = 0.0f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int m = 0; m < 4; ++m) most = fmaxf(most, fabsf(score[n][j][m]));
                }
                if (most <= p.cap_near) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int m = 0; m < 4; ++m) score[n][j][m] = capped_near(p, score[n][j][m]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            const float s = score[n][j][m];
                            score[n][j][m] = fabsf(s) <= p.cap_near ? capped_near(p, s) : capped_far(p, s);
                        }
                    }
                }
            }
        }
        if (!whole) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    if (counts(key + 16 * j + g + 8 * m, j)) continue;
#pragma unroll
                    for (int n = 0; n < kCols; ++n) score[n][j][2 * m] = score[n][j][2 * m + 1] = -INFINITY;
                }
            }
        }
        // The weights are 2^(score - top), where top is the largest score so far less `headroom`, or up to kSlack less: as large as
        // fp16 allows for their products with the values' scales, so that small ones keep their digits.  Scales too large for
        // that much, and scores, renew it.
        float high[kCols][2];
        bool renew = false;
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                high[n][m] = fmaxf(fmaxf(score[n][0][m], score[n][0][2 + m]), fmaxf(score[n][1][m], score[n][1][2 + m]));
                renew |= high[n][m] > top[n][m] + (headroom + kSlack);
            }
        }
        uint32_t vs[2][2][kGroups / 2];                         // scales of the values of keys g and g + 8
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                load_words<kGroups / 2>(stage + j * C::kBytes + C::kValueScales + (g + 8 * m) * 2 * kGroups, vs[j][m]);
                if (!whole && !counts(key + 16 * j + g + 8 * m, j)) {       // whatever the page holds there
#pragma unroll
                    for (int t = 0; t < kGroups / 2; ++t) vs[j][m][t] = 0;
                }
#pragma unroll
                for (int t = 0; t < kGroups / 2; ++t) renew |= !__hblt2(*reinterpret_cast<const __half2*>(&vs[j][m][t]), scale_limit);
            }
        }
        if (__any_sync(0xFFFFFFFFu, renew)) {
            unsigned most = 0;                                  // the largest scale, as its bits
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
#pragma unroll
                    for (int t = 0; t < kGroups / 2; ++t) most = max(most, max(vs[j][m][t] & 0x7FFFu, vs[j][m][t] >> 16 & 0x7FFFu));
                }
            }
            most = __reduce_max_sync(0xFFFFFFFFu, most);        // below 2^(its exponent - 14)
            const float before = headroom;
            headroom = fminf(headroom, fmaxf(28.0f - static_cast<float>(most >> 10), 0.0f));
            scale_limit = __float2half2_rn(exp2f(14.0f - headroom));
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    float largest = high[n][m];
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) largest = fmaxf(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, d));
                    const float next = fmaxf(top[n][m] + before, largest) - headroom, f = exp2_of(top[n][m] - next);
                    top[n][m] = next;
                    weight[n][m] *= f;
#pragma unroll
                    for (int t = 0; t < 2 * kGroups; ++t) acc[n][t][m] *= f, acc[n][t][2 + m] *= f;
                }
            }
        }
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    score[n][j][m] = exp2_of(score[n][j][m] - top[n][m & 1]);
                    weight[n][m & 1] += score[n][j][m];
                }
            }
        }
        const uint32_t mine = g & 1 ? 0x7632 : 0x5410;          // the lane's half of a word: dimensions 4 g .. 4 g + 3 of the scale's 32
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t v[4][kGroups];                             // of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
            for (int m = 0; m < 4; ++m)
                load_words<kGroups>(stage + j * C::kBytes + C::kValues + (2 * c + (m & 1) + 8 * (m >> 1)) * C::kValueRow + (g >> 1) * 4 * kGroups, v[m]);
#pragma unroll
            for (int t = 0; t < kGroups; ++t) {
                const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&vs[j][0][t / 2])), f1 = __half22float2(*reinterpret_cast<const __half2*>(&vs[j][1][t / 2]));
                const float s0 = t & 1 ? f0.y : f0.x, s1 = t & 1 ? f1.y : f1.x;
                uint32_t ab[4], cd[4];
                pairs_of(__byte_perm(v[0][t], v[1][t], mine), ab);
                pairs_of(__byte_perm(v[2][t], v[3][t], mine), cd);
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
                    const __half2 low = __floats2half2_rn(score[n][j][0] * s0, score[n][j][1] * s0), up = __floats2half2_rn(score[n][j][2] * s1, score[n][j][3] * s1);
                    const uint32_t lo = transpose8x8(*reinterpret_cast<const uint32_t*>(&low)), hi = transpose8x8(*reinterpret_cast<const uint32_t*>(&up));
                    dev::mma_f16(acc[n][2 * t], ab[0], ab[1], cd[0], cd[1], lo, hi);
                    dev::mma_f16(acc[n][2 * t + 1], ab[2], ab[3], cd[2], cd[3], lo, hi);
                }
            }
        }
    }

    // the warps' sums, joined
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    float* sums = reinterpret_cast<float*>(rings + w * kRing);
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) weight[n][i] += __shfl_xor_sync(0xFFFFFFFFu, weight[n][i], d);
            const int row = 8 * n + 2 * c + i;
            if (g == 0) warp_stats[w * kRows + row] = make_float2(top[n][i], weight[n][i]);
            float* to = sums + row * kDim;
#pragma unroll
            for (int j = 0; j < 2 * kGroups; ++j) {
                const int d = 32 * (j / 2) + 4 * g + 2 * (j % 2);
                *reinterpret_cast<float2*>(to + d) = make_float2(acc[n][j][i], acc[n][j][2 + i]);
            }
        }
    }
}

// A CTA's sums of four neighbouring dimensions of a row, from its warps'; (maximum, weight) in `stat`.
template <int kGroups, int kCols>
__device__ __forceinline__ float4 join_warps(const unsigned char* rings, const float2* warp_stats, int row, int d, float2& stat) {
    using S = Shape<kGroups, kCols>;
    float m = kLowest, wt = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) m = fmaxf(m, warp_stats[i * S::kRows + row].x);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        const float2 st = warp_stats[i * S::kRows + row];
        const float f = exp2_of(st.x - m);
        const float4 v = *reinterpret_cast<const float4*>(rings + i * S::kRing + (row * S::kDim + d) * 4);
        wt += st.y * f;
        sum.x += v.x * f, sum.y += v.y * f, sum.z += v.z * f, sum.w += v.w * f;
    }
    stat = make_float2(m, wt);
    return sum;
}

template <int kGroups, int kCols>
__global__ void __launch_bounds__(kThreads, Shape<kGroups, kCols>::kCtasOfSm) attn_kernel(const AttnParams p) {
    using S = Shape<kGroups, kCols>;
    constexpr int kDim = S::kDim, kRows = S::kRows, kRing = S::kRing;
    extern __shared__ float4 shared[];
    unsigned char* rings = reinterpret_cast<unsigned char*>(shared);                    // [warp]: the stages, then sums [kRows][kDim]
    float2* warp_stats = reinterpret_cast<float2*>(rings + kWarps * kRing);             // [warp][kRows]
    int* warp_sums = reinterpret_cast<int*>(warp_stats + kWarps * kRows);
    int* first = warp_sums + kWarps;
    dev::programmatic_start();
    scan_units(p, first, warp_sums);
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {         // requests without keys
        if (first[b] != first[b + 1]) continue;
        const int columns = p.heads * p.group * kDim;
        for (int i = threadIdx.x; i < columns; i += kThreads) p.y[b * p.ldy + i] = __ushort_as_half(0);
        if (p.mask != nullptr)
            for (int i = threadIdx.x; i < columns / 32; i += kThreads) p.mask[b * p.mask_stride + i] = 0.0f <= p.thr ? 0u : 0xFFFFFFFFu;
        if (p.by_triple)
            for (int i = threadIdx.x; i < p.heads * p.row_blocks; i += kThreads) p.open[b * p.heads * p.row_blocks + i].x = -1;
    }
    if (!p.by_triple && threadIdx.x == 0) p.open[blockIdx.x].x = -1;
    const int total = first[p.B], ctas = min(static_cast<int>(gridDim.x), total);       // so that no CTA between two others has nothing
    if (static_cast<int>(blockIdx.x) >= ctas) return;
    const int begin = run_start(total, ctas, blockIdx.x), stop = run_start(total, ctas, blockIdx.x + 1);
    int pieces = 0;
    for (int u = begin; u < stop;) {
        int b = 0;                                              // the last request that does not begin behind u: it has keys
        for (int lo = 0, hi = p.B - 1; lo <= hi;) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= u) b = mid, lo = mid + 1;
            else hi = mid - 1;
        }
        const Span span = span_of(p, b);
        const int length = triple_length(span.units), triple = (u - first[b]) / length, at = (u - first[b]) % length;
        const int start = u - at;                               // of the triple
        const int off = max(0, at - kStart), count = max(0, min(length, stop - start) - kStart) - off;
        u = min(start + length, stop);
        if (count <= 0) continue;                               // the run ends before the triple's first unit
        const int h = triple / p.row_blocks, row0 = triple % p.row_blocks * kRows, rows = min(kRows, p.group - row0);
        const int k0 = span.low + off * kUnit, k1 = min(span.end, k0 + count * kUnit);
        attend<kGroups, kCols>(p, b, h, row0, k0, k1, span.end, rings, warp_stats);
        __syncthreads();
        const bool all = count == span.units;
        const int slot = 2 * blockIdx.x + (pieces > 0 ? 1 : 0); // what is not whole is the first piece of a run or the last
        ++pieces;
        for (int e = threadIdx.x; e < rows * kDim / 4; e += kThreads) {       // four neighbours to a thread
            const int row = e / (kDim / 4), d = e % (kDim / 4) * 4;
            float2 stat;
            const float4 sum = join_warps<kGroups, kCols>(rings, warp_stats, row, d, stat);
            if (all) {
                store_result(p, b, static_cast<int64_t>(h * p.group + row0 + row) * kDim + d, sum, stat.y);
            } else {
                *reinterpret_cast<float4*>(p.sums + (static_cast<int64_t>(slot) * kRows + row) * kDim + d) = sum;
                if (d == 0) p.stats[slot * kRows + row] = stat;
            }
        }
        if (threadIdx.x == 0 && off == 0 && (p.by_triple || !all))        // the CTAs with the rest follow this one
            p.open[p.by_triple ? b * p.heads * p.row_blocks + triple : blockIdx.x] =
                make_int4(all ? -1 : b, triple, slot, static_cast<int>(((static_cast<int64_t>(start) + length) * ctas - 1) / total));
        __syncthreads();
    }
}

// The form for few triples of few keys: a cluster of CTAs to a triple, an eighth of its keys each, whose sums meet through
// distributed shared memory.  No scratch memory, no second kernel.
constexpr int kCluster = 8;

template <int kGroups, int kCols>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, Shape<kGroups, kCols>::kCtasOfSm) attn_cluster_kernel(const AttnParams p) {
    using S = Shape<kGroups, kCols>;
    constexpr int kDim = S::kDim, kRows = S::kRows, kRing = S::kRing;
    extern __shared__ float4 shared[];
    unsigned char* rings = reinterpret_cast<unsigned char*>(shared);
    float2* warp_stats = reinterpret_cast<float2*>(rings + kWarps * kRing);
    float2* stats = warp_stats + kWarps * kRows;                // [kRows], read by the whole cluster, as the first warp's sums are
    dev::programmatic_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int cta = blockIdx.x % kCluster, place = blockIdx.x / kCluster, triples = p.heads * p.row_blocks, b = place / triples, triple = place % triples;
    const int h = triple / p.row_blocks, row0 = triple % p.row_blocks * kRows, rows = min(kRows, p.group - row0);
    const Span span = span_of(p, b);
    const int steps = (span.end - span.low + 31) / 32;          // of 32 keys
    const int k0 = span.low + 32 * (steps * cta / kCluster), k1 = min(span.end, span.low + 32 * (steps * (cta + 1) / kCluster));
    attend<kGroups, kCols>(p, b, h, row0, k0, k1, span.end, rings, warp_stats);
    __syncthreads();
    for (int e = threadIdx.x; e < rows * kDim / 4; e += kThreads) {
        const int row = e / (kDim / 4), d = e % (kDim / 4) * 4;
        float2 stat;
        const float4 sum = join_warps<kGroups, kCols>(rings, warp_stats, row, d, stat);
        *reinterpret_cast<float4*>(rings + (row * kDim + d) * 4) = sum;      // nobody else reads or writes the first warp's there
        if (d == 0) stats[row] = stat;
    }
    cluster.sync();
    const int e = cta * kThreads + threadIdx.x;
    static_assert(kRows * kDim / 4 <= kCluster * kThreads, "a thread of the cluster for every four results");
    if (e < rows * kDim / 4) {
        const int row = e / (kDim / 4), d = e % (kDim / 4) * 4;
        float m = kLowest, wt = 0.0f;
        float2 st[kCluster];
        float4 v[kCluster], sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {
            st[i] = cluster.map_shared_rank(stats, i)[row];
            v[i] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(rings, i) + (row * kDim + d) * 4);
            m = fmaxf(m, st[i].x);
        }
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {
            const float f = exp2_of(st[i].x - m);
            wt += st[i].y * f;
            sum.x += v[i].x * f, sum.y += v[i].y * f, sum.z += v[i].z * f, sum.w += v[i].w * f;
        }
        store_result(p, b, static_cast<int64_t>(h * p.group + row0 + row) * kDim + d, sum, wt);
    }
    cluster.sync();                                             // nobody reads this CTA's sums any more
}

// Joins the partial sums of a triple that several CTAs have, in the order of its keys: a row of it to a CTA, whose groups of lanes
// take every kParts-th sum.
constexpr int kJoinThreads = 256;

template <int kGroups, int kCols>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const AttnParams p) {
    constexpr int kDim = 32 * kGroups, kRows = 8 * kCols, kLanes = kDim / 4, kParts = kJoinThreads / kLanes;
    __shared__ __align__(16) float part[kParts][kDim];
    __shared__ float2 stat[kParts];
    dev::programmatic_start();
    const int4 open = p.open[blockIdx.x];
    if (open.x < 0) return;
    const int b = open.x, h = open.y / p.row_blocks, row = blockIdx.y, head = open.y % p.row_blocks * kRows + row;
    if (head >= p.group) return;
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
    store_result(p, b, static_cast<int64_t>(h * p.group + head) * kDim + d, sum, wt);
}

// The same for few triples of many sums each, where it is all latency: the first kAhead sums of a group are asked for together with
// all maxima.
// CTAs to a triple from which on this form is taken (us with it and with the other, requests of 16384 keys, 64 and 8 heads: 74 CTAs
// 23.8 : 25.9, 37 28.0 : 30.0, 25 33.0 : 34.0, 18 38.2 : 38.2, 15 44.3 : 42.3, 9 58.7 : 54.6, 1.5 240.9 : 219; 16 and 1 heads: 592 CTAs 21.8 :
// 26.3, 37 34.1 : 36.1, 25 44.3 : 42.3, 12 64.9 : 60.7).
constexpr int kJoinFew = 16;
constexpr int kJoinChunk = kJoinThreads;                        // sums whose maxima and weights are in shared memory at a time

template <int kGroups, int kCols>
__global__ void __launch_bounds__(kJoinThreads) attn_join_few_kernel(const AttnParams p) {
    constexpr int kDim = 32 * kGroups, kRows = 8 * kCols, kLanes = kDim / 4, kParts = kJoinThreads / kLanes, kAhead = 12;
    __shared__ __align__(16) float part[kParts][kDim];
    __shared__ float2 stats[kJoinChunk];
    __shared__ float warp_tops[kJoinThreads / 32], weights[kParts];
    dev::programmatic_start();
    const int4 open = p.open[blockIdx.x];
    if (open.x < 0) return;
    const int b = open.x, h = open.y / p.row_blocks, row = blockIdx.y, head = open.y % p.row_blocks * kRows + row;
    if (head >= p.group) return;
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
    store_result(p, b, static_cast<int64_t>(h * p.group + head) * kDim + d, sum, wt);
}

template <int kGroups, int kCols>
size_t attn_shared_bytes(int B) { return kWarps * (Shape<kGroups, kCols>::kRing + 8 * kCols * sizeof(float2) + sizeof(int)) + (B + 1) * sizeof(int); }

template <int kGroups, int kCols>
size_t attn_cluster_bytes() { return kWarps * Shape<kGroups, kCols>::kRing + (kWarps + 1) * 8 * kCols * sizeof(float2); }

// Up to here a cluster to a triple, where all of them fit the GPU at once (64 query and 8 key heads, in a graph, us, cluster against
// line: 1 request of 1000 keys 10.2 against 15.6, of 8000 18.4 : 21.8, of 12000 20.5 : 23.8, of 16000 24.6 : 23.9, of 32000 38.9 : 27.9; 2 of
// 8000 22.5 : 23.8, of 12000 26.6 : 26.0; 9 of 8000 38.9 : 40.2, of 12000 51.2 : 48.4, the others of a sixteenth of it 24.6 : 27.9).  What
// decides is the longest that the table allows: a request's own length is only known on the device.
constexpr int kClusterKeys = 8192;

template <int kGroups, int kCols>
spdp_status launch_form(AttnParams p, int device, int sms, cudaStream_t s) {
    constexpr int kDim = 32 * kGroups, kRows = 8 * kCols;
    static std::mutex mu;
    static int resident[64] = {};                               // CTAs of an SM
    int per_sm;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (resident[device] == 0) {
            SPDP_CUDA_TRY(cudaFuncSetAttribute(attn_kernel<kGroups, kCols>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(attn_shared_bytes<kGroups, kCols>(kMostRequests))));
            SPDP_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident[device], attn_kernel<kGroups, kCols>, kThreads,
                                                                        attn_shared_bytes<kGroups, kCols>(64)));
            SPDP_CUDA_TRY(cudaFuncSetAttribute(attn_cluster_kernel<kGroups, kCols>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(attn_cluster_bytes<kGroups, kCols>())));
        }
        per_sm = resident[device] > 0 ? resident[device] : 1;
    }
    const int triples = p.heads * p.row_blocks;
    const int64_t longest = p.window > 0 && p.window < p.table_pages << p.page_shift ? p.window : p.table_pages << p.page_shift;
    if (longest <= kClusterKeys && static_cast<int64_t>(p.B) * triples * kCluster <= static_cast<int64_t>(per_sm) * sms) {
        SPDP_CUDA_TRY(launch_programmatic(attn_cluster_kernel<kGroups, kCols>, dim3(static_cast<unsigned>(p.B * triples * kCluster)), kThreads,
                                          attn_cluster_bytes<kGroups, kCols>(), s, p));
        return SPDP_OK;
    }
    // no more CTAs than there can be units
    const int64_t most = p.B * (((p.table_pages << p.page_shift) + kUnit - 1) / kUnit) * triples;
    const int ctas = static_cast<int>(most < static_cast<int64_t>(per_sm) * sms ? most : per_sm * sms);
    const size_t sums = 2ull * ctas * kRows * kDim * sizeof(float), stats = 2ull * ctas * kRows * sizeof(float2);
    void* scratch = nullptr;
    spdp_status st = scratch_alloc(device, sums + stats + ctas * sizeof(int4), s, &scratch);
    if (st != SPDP_OK) return st;
    p.sums = static_cast<float*>(scratch);
    p.stats = reinterpret_cast<float2*>(static_cast<char*>(scratch) + sums);
    p.by_triple = static_cast<int64_t>(p.B) * triples <= ctas;
    const int places = p.by_triple ? p.B * triples : ctas;
    p.open = reinterpret_cast<int4*>(static_cast<char*>(scratch) + sums + stats);
    cudaError_t e = launch_programmatic(attn_kernel<kGroups, kCols>, dim3(static_cast<unsigned>(ctas)), kThreads, attn_shared_bytes<kGroups, kCols>(p.B), s, p);
    if (e == cudaSuccess) e = launch_programmatic(ctas >= kJoinFew * places ? attn_join_few_kernel<kGroups, kCols> : attn_join_kernel<kGroups, kCols>, dim3(static_cast<unsigned>(places), static_cast<unsigned>(p.group < kRows ? p.group : kRows)), kJoinThreads, 0, s, p);
    const cudaError_t freed = cudaFreeAsync(scratch, s);
    SPDP_CUDA_TRY(e);
    SPDP_CUDA_TRY(freed);
    return SPDP_OK;
}

template <int kGroups>
spdp_status launch_groups(AttnParams p, int device, int sms, cudaStream_t s) {
    if (p.group <= 8) {
        p.row_blocks = 1;
        return launch_form<kGroups, 1>(p, device, sms, s);
    }
    p.row_blocks = (p.group + 15) / 16;
    return launch_form<kGroups, 2>(p, device, sms, s);
}

int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

}  // namespace

spdp_status launch_kv4_store(const Kv4StoreCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    StoreParams p = {};
    p.k = call.k, p.v = call.v, p.slot = call.slot, p.cache = call.cache, p.k_values = call.k_values, p.v_values = call.v_values;
    p.ldk = call.ldk, p.ldv = call.ldv, p.ldk_values = call.ldk_values, p.ldv_values = call.ldv_values, p.N = call.N, p.pages = call.pages;
    p.heads = call.kv_heads, p.dim = call.head_dim, p.page_shift = log2_of(call.page_tokens);
    const bool f32 = call.vdt == SPDP_Y_F32;
    const bool wide = rows_aligned16(p.k, p.ldk, 2) && rows_aligned16(p.v, p.ldv, f32 ? 4 : 2) && rows_aligned16(p.k_values, p.ldk_values, 2) &&
                      rows_aligned16(p.v_values, p.ldv_values, 2);
    p.row_shift = log2_of(p.dim / 8);
    SPDP_CUDA_TRY(f32 ? (wide ? launch_store<float, true>(p, sms, s) : launch_store<float, false>(p, sms, s))
                      : (wide ? launch_store<__half, true>(p, sms, s) : launch_store<__half, false>(p, sms, s)));
    return SPDP_OK;
}

spdp_status launch_attn_kv4(const Kv4AttnCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    AttnParams p = {};
    p.q = call.q, p.cache = call.cache, p.table = call.table, p.length = call.length, p.y = call.y, p.mask = call.mask;
    p.ldq = call.ldq, p.ldy = call.ldy, p.table_stride = call.table_stride, p.table_pages = call.table_pages, p.mask_stride = call.mask_stride, p.pages = static_cast<unsigned>(call.pages);
    p.B = static_cast<int>(call.B), p.heads = call.kv_heads, p.group = call.q_heads / call.kv_heads, p.page_shift = log2_of(call.page_tokens);
    constexpr float kLog2e = 1.4426950408889634f;
    p.scale = call.scale * kLog2e;
    p.cap = call.cap * kLog2e;
    p.cap_inv = call.cap > 0.0f ? fminf(1.0f / p.cap, FLT_MAX) : 0.0f;         // never Inf, for a score may be 0
    p.cap_near = 0.25f * p.cap;
    p.window = call.window, p.thr = call.thr;
    p.wide_q = rows_aligned16(p.q, p.ldq, 2), p.wide_y = rows_aligned16(p.y, p.ldy, 2);
    switch (call.head_dim) {
        case 64: return launch_groups<2>(p, device, sms, s);
        case 128: return launch_groups<4>(p, device, sms, s);
        default: return launch_groups<8>(p, device, sms, s);
    }
}

}  // namespace spdp
