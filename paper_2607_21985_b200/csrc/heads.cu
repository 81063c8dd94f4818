// Norms of the query and key heads and their rotation by positions, in one pass over what a q/k/v projection left: a head x
// of D values becomes x / sqrt(mean x^2 + eps) * weight, and the first 2 R of its values are turned in pairs by the angles
// pos[axis of pair i] * inv_freq[i].  Heads are read once and written once (6 bytes a value from 32-bit projections, 4 from
// 16-bit ones): bound by those bytes, for a single token by latency.
//
// A CTA takes one token and a share of its heads.  The token's sines and cosines are computed once, into shared memory, and
// serve all heads.  An angle is formed in 64 bits and in turns, so that whole turns drop out exactly: at position 10^6 a 32-bit
// angle is off by up to 0.03.  A lane holds both members of its pairs; 8 pairs to a lane where alignment lets it load 16 bytes
// at once, so 8 lanes share a head of 128 and the sum of squares takes 3 exchanges.
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

template <typename T, int kPairs>
__device__ __forceinline__ void load(const T* at, float (&x)[kPairs]) {
    if constexpr (kPairs == 8) dev::load_floats<T, true>(at, x);
    else if constexpr (sizeof(T) == 2) x[0] = __half2float(*at);
    else x[0] = *at;
}

template <int kPairs>
__device__ __forceinline__ void store(__half* at, const float (&x)[kPairs]) {
    if constexpr (kPairs == 8) dev::store_halves<true>(at, x);
    else *at = __float2half_rn(x[0]);
}

// kPairs = 8: 16-byte accesses, D / 16 lanes to a head.  kPairs = 1: any even D up to 256 and any alignment, a head takes up to
// 32 lanes and four rounds of them.
template <typename T, int kPairs, bool kAdjacent>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const Params p) {
    constexpr int kRounds = kPairs == 1 ? kMostDim / 2 / 32 : 1;
    __shared__ float2 turn[kMostDim / 2];
    dev::programmatic_start();
    const int64_t n = blockIdx.x;
    const int half = p.dim / 2, heads = p.q_heads + p.kv_heads;
    const int lane = threadIdx.x & (p.lanes - 1), slots = blockDim.x >> p.shift;
    // The lane's pairs, the same in every head.  Members: neighbours, or as far apart as the pairs that turn; what does not turn is
    // split in two the same way.
    int at[kRounds][2], pair[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = (r * p.lanes + lane) * kPairs;                // the lane's first pair
        pair[r] = i < half ? i : -1;
        if (kAdjacent) at[r][0] = 2 * i, at[r][1] = 2 * i + kPairs;
        else if (i < p.pairs) at[r][0] = i, at[r][1] = i + p.pairs;
        else at[r][0] = i + p.pairs, at[r][1] = i + half;
    }
    float x[kRounds][2][kPairs];
    auto fetch = [&](int h) {
        if (h >= heads) return;
        const T* from = h < p.q_heads ? static_cast<const T*>(p.q) + n * p.ldq + h * p.dim : static_cast<const T*>(p.k) + n * p.ldk + (h - p.q_heads) * p.dim;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
                if (pair[r] >= 0) load<T, kPairs>(from + at[r][m], x[r][m]);
        }
    };
    int h = blockIdx.y * slots + (threadIdx.x >> p.shift);
    fetch(h);                                                       // on its way while the angles are formed
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
        float2 cs = make_float2(1.0f, 0.0f);
        if (i < p.pairs) {
            int a = 0;
            while (a < p.axes - 1 && i >= p.ends[a]) ++a;
            const double turns = static_cast<double>(p.pos[a * p.pos_stride + n]) * static_cast<double>(p.inv_freq[i]) * 0.15915494309189535;  // 1 / (2 pi)
            sincospif(2.0f * static_cast<float>(turns - rint(turns)), &cs.y, &cs.x);
        }
        turn[i] = cs;
    }
    __syncthreads();
    for (int rounds = (heads - blockIdx.y * slots + gridDim.y * slots - 1) / (gridDim.y * slots); rounds > 0; --rounds) {      // the same for all threads
        const bool is_q = h < p.q_heads;
        const __half* weight = is_q ? p.q_weight : p.k_weight;
        float squares = 0.0f, y[kRounds][2][kPairs];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    y[r][m][j] = x[r][m][j];
                    if (h < heads && pair[r] >= 0) squares += y[r][m][j] * y[r][m][j];
                }
            }
        }
        __half* to = is_q ? p.q_out + n * p.ldq_out + h * p.dim : p.k_out + n * p.ldk_out + (h - p.q_heads) * p.dim;
        const bool there = h < heads;
        h += gridDim.y * slots;
        fetch(h);
        for (int d = p.lanes / 2; d > 0; d >>= 1) squares += __shfl_xor_sync(0xFFFFFFFFu, squares, d);
        if (!there) continue;
        if (weight != nullptr) {
            const float inv = 1.0f / sqrtf(squares / p.dim + p.eps);
#pragma unroll
            for (int r = 0; r < kRounds; ++r) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    if (pair[r] < 0) continue;
                    float g[kPairs];
                    load<__half, kPairs>(weight + at[r][m], g);
#pragma unroll
                    for (int j = 0; j < kPairs; ++j) y[r][m][j] = y[r][m][j] * inv * g[j];
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (pair[r] < 0) continue;
            // neighbours: a lane's 2 kPairs values are a0 b0 a1 b1 ...; else y[0] holds the first members and y[1] the second
            float* flat = &y[r][0][0];
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const float2 cs = turn[pair[r] + j];
                float& a = flat[kAdjacent ? 2 * j : j];
                float& b = flat[kAdjacent ? 2 * j + 1 : kPairs + j];
                const float ra = a * cs.x - b * cs.y, rb = b * cs.x + a * cs.y;
                a = ra, b = rb;
            }
            store<kPairs>(to + at[r][0], y[r][0]);
            store<kPairs>(to + at[r][1], y[r][1]);
        }
    }
}

template <typename T, int kPairs>
spdp_status launch_form(const Params& p, bool adjacent, int64_t N, int sms, cudaStream_t s) {
    // Rounds of a token's heads, with no more threads than make them equal.  One CTA takes them in turn (and the angles once)
    // where the tokens fill the GPU; else they are dealt out.
    const int heads = p.q_heads + p.kv_heads, rounds = (heads + (kThreads >> p.shift) - 1) / (kThreads >> p.shift);
    const int threads = ((heads + rounds - 1) / rounds * p.lanes + 31) / 32 * 32, slots = threads >> p.shift;
    int64_t shares = (heads + slots - 1) / slots;
    const int64_t enough = (8 * sms + N - 1) / N;
    if (shares > enough) shares = enough;
    const dim3 grid(static_cast<unsigned>(N), static_cast<unsigned>(shares));
    SPDP_CUDA_TRY(adjacent ? launch_programmatic(qk_norm_rope_kernel<T, kPairs, true>, grid, threads, 0, s, p)
                           : launch_programmatic(qk_norm_rope_kernel<T, kPairs, false>, grid, threads, 0, s, p));
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
    if (size == 4)
        return wide ? launch_form<float, 8>(p, call.adjacent, call.N, sms, s) : launch_form<float, 1>(p, call.adjacent, call.N, sms, s);
    return wide ? launch_form<__half, 8>(p, call.adjacent, call.N, sms, s) : launch_form<__half, 1>(p, call.adjacent, call.N, sms, s);
}

}  // namespace spdp
