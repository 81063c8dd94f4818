// Norms of the query and key heads and their rotation by positions, in one pass over what a q/k/v projection left: a head x
// of D values becomes x / sqrt(mean x^2 + eps) * weight, and the first 2 R of its values are turned in pairs by the angles
// pos[axis of pair i] * inv_freq[i].  Heads are read once and written once (6 bytes a value from 32-bit projections, 4 from
// 16-bit ones): bound by those bytes, for a single token by latency.
//
// A CTA takes one token and a share of its heads.  The token's sines and cosines are computed once, into shared memory, and
// serve all heads.  An angle is formed in 64 bits and in turns, so that whole turns drop out exactly: at position 10^6 a 32-bit
// angle is off by up to 0.03.  A lane holds both members of its pairs; 8 pairs to a lane where alignment lets it load 16 bytes
// at once, so 8 lanes share a head of 128 and the sum of squares takes 3 exchanges.
//
// 4096 tokens of 64 and 8 heads of 128 from 32-bit rows: 39 us, 226 MB at 5.8 TB/s.  2547 of 32 and 8 heads of 256, 16-bit: 35 us, 49
// with one kernel for every alignment, whose sines and cosines came from shared memory for each head.
#include "mma_f16.cuh"
#include "spdp_internal.h"

namespace spdp {
namespace {

constexpr int kThreads = 256;
constexpr int kMostDim = 256;
constexpr int kMostAxes = 4;

struct Params {
    const void* q;
    const void* k;
    const __half* q_weight;
    const __half* k_weight;
    const int32_t* pos;
    const float* inv_freq;
    __half* q_out;
    __half* k_out;
    int64_t ldq, ldk, ldq_out, ldk_out, pos_stride;
    int q_heads, kv_heads, dim, pairs;          // pairs that turn
    int axes, ends[kMostAxes];                  // pairs below ends[a] (and not below ends[a - 1]) turn by axis a
    int lanes, shift;                           // lanes of a head, a power of two, and its logarithm
    float eps;
};

// Sine and cosine of a pair's angle for token n; pairs that do not turn have 0 and 1.
__device__ __forceinline__ void turn_of(const Params& p, int64_t n, int i, float& sine, float& cosine) {
    sine = 0.0f, cosine = 1.0f;
    if (i >= p.pairs) return;
    int a = 0;
    while (a < p.axes - 1 && i >= p.ends[a]) ++a;
    const double turns = static_cast<double>(p.pos[a * p.pos_stride + n]) * static_cast<double>(p.inv_freq[i]) * 0.15915494309189535;  // 1 / (2 pi)
    sincospif(2.0f * static_cast<float>(turns - rint(turns)), &sine, &cosine);
}

// Where the two members of pair i are: neighbours, or as far apart as the pairs that turn; what does not turn is split in two the
// same way.  (Neighbours: the first values of `count` pairs, and of the second half of these.)
template <bool kAdjacent>
__device__ __forceinline__ void members_of(const Params& p, int i, int count, int& first, int& second) {
    if (kAdjacent) first = 2 * i, second = 2 * i + count;
    else if (i < p.pairs) first = i, second = i + p.pairs;
    else first = i + p.pairs, second = i + p.dim / 2;
}

// 16-byte accesses: a lane has 8 pairs, D / 16 lanes (rounded up to a power of two) a head.  The sines and cosines of a lane's
// pairs, the same in every head, stay in its registers.
template <typename T, bool kAdjacent>
__global__ void __launch_bounds__(kThreads, 4) qk_norm_rope_wide_kernel(const Params p) {
    __shared__ __align__(16) float sines[kMostDim / 2], cosines[kMostDim / 2];
    dev::programmatic_start();
    const int64_t n = blockIdx.x;
    const int half = p.dim / 2, heads = p.q_heads + p.kv_heads;
    const int lane = threadIdx.x & (p.lanes - 1), slots = blockDim.x >> p.shift, stride = gridDim.y * slots;
    const bool mine = 8 * lane < half;
    int first, second;
    members_of<kAdjacent>(p, 8 * lane, 8, first, second);
    float x[2][8];
    auto fetch = [&](int h) {
        if (h >= heads || !mine) return;
        const T* from = h < p.q_heads ? static_cast<const T*>(p.q) + n * p.ldq + h * p.dim : static_cast<const T*>(p.k) + n * p.ldk + (h - p.q_heads) * p.dim;
        dev::load_floats<T, true>(from + first, x[0]);
        dev::load_floats<T, true>(from + second, x[1]);
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) x[0][j] = x[1][j] = 0.0f;
    int h = blockIdx.y * slots + (threadIdx.x >> p.shift);
    fetch(h);                                                       // on its way while the angles are formed
    for (int i = threadIdx.x; i < half; i += blockDim.x) turn_of(p, n, i, sines[i], cosines[i]);
    __syncthreads();
    float s[8], c[8];
    if (mine) {
        dev::load_floats<float, true>(sines + 8 * lane, s);
        dev::load_floats<float, true>(cosines + 8 * lane, c);
    }
    const float per_value = 1.0f / p.dim;
    const int turning = p.pairs - 8 * lane;                         // of the lane's pairs; the rest stay as they are (an Inf next to 0 turns would leave NaN)
    for (int rounds = (heads - blockIdx.y * slots + stride - 1) / stride; rounds > 0; --rounds, h += stride) {     // the same for all threads
        float squares = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) squares += x[0][j] * x[0][j] + x[1][j] * x[1][j];
        for (int d = p.lanes / 2; d > 0; d >>= 1) squares += __shfl_xor_sync(0xFFFFFFFFu, squares, d);
        if (h >= heads || !mine) continue;
        const bool is_q = h < p.q_heads;
        const __half* weight = is_q ? p.q_weight : p.k_weight;
        float y[2][8];
        if (weight != nullptr) {
            const float inv = rsqrtf(squares * per_value + p.eps);
            dev::load_floats<__half, true>(weight + first, y[0]);
            dev::load_floats<__half, true>(weight + second, y[1]);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[0][j] *= x[0][j] * inv, y[1][j] *= x[1][j] * inv;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[0][j] = x[0][j], y[1][j] = x[1][j];
        }
        fetch(h + stride);
        // neighbours: a lane's 16 values are a0 b0 a1 b1 ...; else y[0] holds the first members and y[1] the second
        float* flat = &y[0][0];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!(kAdjacent ? j < turning : turning > 0)) continue;
            float& a = flat[kAdjacent ? 2 * j : j];
            float& b = flat[kAdjacent ? 2 * j + 1 : 8 + j];
            const float ra = a * c[j] - b * s[j], rb = b * c[j] + a * s[j];
            a = ra, b = rb;
        }
        __half* to = is_q ? p.q_out + n * p.ldq_out + h * p.dim : p.k_out + n * p.ldk_out + (h - p.q_heads) * p.dim;
        dev::store_halves<true>(to + first, y[0]);
        dev::store_halves<true>(to + second, y[1]);
    }
}

// Any even D up to 256 and any alignment: a lane has a pair in each of up to four rounds, up to 32 lanes a head.
template <typename T, bool kAdjacent>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const Params p) {
    constexpr int kRounds = kMostDim / 2 / 32;
    __shared__ float sines[kMostDim / 2], cosines[kMostDim / 2];
    dev::programmatic_start();
    const int64_t n = blockIdx.x;
    const int half = p.dim / 2, heads = p.q_heads + p.kv_heads;
    const int lane = threadIdx.x & (p.lanes - 1), slots = blockDim.x >> p.shift, stride = gridDim.y * slots;
    for (int i = threadIdx.x; i < half; i += blockDim.x) turn_of(p, n, i, sines[i], cosines[i]);
    __syncthreads();
    int h = blockIdx.y * slots + (threadIdx.x >> p.shift);
    for (int rounds = (heads - blockIdx.y * slots + stride - 1) / stride; rounds > 0; --rounds, h += stride) {     // the same for all threads
        const bool there = h < heads, is_q = h < p.q_heads;
        const T* from = is_q ? static_cast<const T*>(p.q) + n * p.ldq + h * p.dim : static_cast<const T*>(p.k) + n * p.ldk + (h - p.q_heads) * p.dim;
        const __half* weight = is_q ? p.q_weight : p.k_weight;
        float x[kRounds][2], squares = 0.0f;
        int at[kRounds][2];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = r * p.lanes + lane;
            members_of<kAdjacent>(p, i, 1, at[r][0], at[r][1]);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                x[r][m] = 0.0f;
                if (there && i < half) {
                    if constexpr (sizeof(T) == 2) x[r][m] = __half2float(from[at[r][m]]);
                    else x[r][m] = from[at[r][m]];
                }
                squares += x[r][m] * x[r][m];
            }
        }
        for (int d = p.lanes / 2; d > 0; d >>= 1) squares += __shfl_xor_sync(0xFFFFFFFFu, squares, d);
        if (!there) continue;
        const float inv = rsqrtf(squares / p.dim + p.eps);
        __half* to = is_q ? p.q_out + n * p.ldq_out + h * p.dim : p.k_out + n * p.ldk_out + (h - p.q_heads) * p.dim;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = r * p.lanes + lane;
            if (i >= half) continue;
            if (weight != nullptr) {
#pragma unroll
                for (int m = 0; m < 2; ++m) x[r][m] = x[r][m] * inv * __half2float(weight[at[r][m]]);
            }
            const bool turns = i < p.pairs;
            to[at[r][0]] = __float2half_rn(turns ? x[r][0] * cosines[i] - x[r][1] * sines[i] : x[r][0]);
            to[at[r][1]] = __float2half_rn(turns ? x[r][1] * cosines[i] + x[r][0] * sines[i] : x[r][1]);
        }
    }
}

template <typename T>
spdp_status launch_form(const Params& p, bool wide, bool adjacent, int64_t N, int sms, cudaStream_t s) {
    // Rounds of a token's heads, with no more threads than make them equal.  One CTA takes them in turn (and the angles once)
    // where the tokens fill the GPU; else they are dealt out.
    const int heads = p.q_heads + p.kv_heads, rounds = (heads + (kThreads >> p.shift) - 1) / (kThreads >> p.shift);
    const int threads = ((heads + rounds - 1) / rounds * p.lanes + 31) / 32 * 32, slots = threads >> p.shift;
    int64_t shares = (heads + slots - 1) / slots;
    const int64_t enough = (8 * sms + N - 1) / N;
    if (shares > enough) shares = enough;
    const dim3 grid(static_cast<unsigned>(N), static_cast<unsigned>(shares));
    SPDP_CUDA_TRY(launch_programmatic(wide ? (adjacent ? qk_norm_rope_wide_kernel<T, true> : qk_norm_rope_wide_kernel<T, false>)
                                           : (adjacent ? qk_norm_rope_kernel<T, true> : qk_norm_rope_kernel<T, false>),
                                      grid, threads, 0, s, p));
    return SPDP_OK;
}

}  // namespace

spdp_status launch_qk_norm_rope(const HeadsCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    Params p = {};
    p.q = call.q, p.k = call.k, p.q_weight = call.q_weight, p.k_weight = call.k_weight, p.pos = call.pos, p.inv_freq = call.inv_freq;
    p.q_out = call.q_out, p.k_out = call.k_out, p.ldq = call.ldq, p.ldk = call.ldk, p.ldq_out = call.ldq_out, p.ldk_out = call.ldk_out;
    p.pos_stride = call.pos_stride, p.q_heads = call.q_heads, p.kv_heads = call.kv_heads, p.dim = call.head_dim, p.pairs = call.pairs;
    p.axes = call.axes, p.eps = call.eps;
    for (int a = 0, end = 0; a < call.axes; ++a) p.ends[a] = end += call.sections[a];
    const int64_t size = call.dt == SPDP_Y_F32 ? 4 : 2;
    const bool rows = (call.q_heads == 0 || (rows_aligned16(call.q, call.ldq, size) && rows_aligned16(call.q_out, call.ldq_out, 2) && rows_aligned16(call.q_weight, 0, 0))) &&
                      (call.kv_heads == 0 || (rows_aligned16(call.k, call.ldk, size) && rows_aligned16(call.k_out, call.ldk_out, 2) && rows_aligned16(call.k_weight, 0, 0)));
    const bool wide = rows && call.head_dim % 16 == 0 && (call.adjacent || call.pairs % 8 == 0);
    const int needed = wide ? call.head_dim / 16 : call.head_dim / 2;
    for (p.lanes = 1, p.shift = 0; p.lanes < needed && p.lanes < 32; p.lanes *= 2) ++p.shift;
    return size == 4 ? launch_form<float>(p, wide, call.adjacent, call.N, sms, s) : launch_form<__half>(p, wide, call.adjacent, call.N, sms, s);
}

}  // namespace spdp
