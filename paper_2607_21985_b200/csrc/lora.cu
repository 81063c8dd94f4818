// Low-rank adapters of many requests beside a shared projection: y_n = base_n + s_a B_a (A_a x_n), where a is the adapter of
// token n.  Folding B A into a statically pruned W would fill its zeros, so an adapter of a packed layer has to stay beside it.
//
// The work is the bytes: x, base and y once, the weights of the adapters in use; the products are a few times the rank per byte.
// One launch does both products.  A cluster of 8 CTAs takes 32 consecutive tokens and one adapter among them: each CTA
// multiplies an eighth of K (its warps split that again), the partial sums meet through distributed shared memory in a fixed
// order, and each CTA then multiplies the rank-long vectors into its share of the output rows.  So the vectors between the
// two products never leave the chip, there is no workspace, and x, base and y cross memory once whatever N is.  Where there are
// few tokens several clusters share a tile: one to an adapter, or, past that, each with a part of the output rows, the
// (small) first product done by each of them.
//
// Both products run on mma.sync with tokens as the 8 columns and weight rows as the 16 rows, fragments loaded straight from
// memory: a lane holds 8 consecutive elements of a row, the same on both sides.  The vectors between the products are kept
// in fp16 for the second one, scaled per token by a power of two (so that neither end of the range is lost): one rounding of
// 2^-12 on a term that is added to a 16-bit result; for 32-bit results a second fp16 number holds what the first one lost.
#include <cooperative_groups.h>

#include <mutex>

#include "mma_f16.cuh"
#include "spdp_internal.h"

namespace cg = cooperative_groups;

namespace spdp {
namespace {

constexpr int kTok = 32;            // tokens of a tile: 4 column blocks of 8
constexpr int kTokPad = 40;         // floats from one rank to the next in shared memory: the fragments' stores meet no bank twice
constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kCluster = 8;
constexpr int kOut = 64;            // output rows of a warp's block
constexpr int kBlocksOfCluster = kCluster * kWarps;

struct Params {
    const __half* X;
    const int32_t* adapter;
    const __half* A;
    const __half* B;
    const int32_t* ranks;
    const float* scales;
    const void* base;
    void* Y;
    int64_t ldx, lda, stride_a, ldb, stride_b, ldbase, ldy;
    int N, K, M, count, rank;
    int per_tile;                   // clusters of a tile
    bool wide_x, wide_a, wide_b, wide_y;
};

__host__ __device__ inline int padded_rank(int rank) { return (rank + 31) & ~31; }

template <int kRankTiles>
struct Layout {                     // shared memory, in floats
    static __host__ __device__ int sums(int rank) {
        const int warps = kWarps * 16 * kRankTiles, all = padded_rank(rank);
        return (warps > all ? warps : all) * kTokPad;
    }
    static __host__ __device__ int part(int rank) { return padded_rank(rank) * kTokPad; }
    static __host__ __device__ int row(int rank) { return padded_rank(rank) + 8; }       // halves of a token's vector
    static __host__ __device__ size_t bytes(int rank, bool f32) {
        return 4u * (sums(rank) + part(rank) + (kWarps + 1) * kTok) + 2u * kTok * row(rank) * (f32 ? 2 : 1);
    }
};

template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 2) return __half2float(v);
    else return v;
}

// o[8] to y, on top of base's eight values; `left` of them exist.
template <typename T>
__device__ __forceinline__ void add_store(const T* base, T* y, const float (&o)[8], int left, bool wide) {
    if (wide && left >= 8) {
        if constexpr (sizeof(T) == 2) {
            const uint4 b = *reinterpret_cast<const uint4*>(base);
            const uint32_t in[4] = {b.x, b.y, b.z, b.w};
            uint32_t out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&in[i]));
                const __half2 r = __floats2half2_rn(f.x + o[2 * i], f.y + o[2 * i + 1]);
                out[i] = *reinterpret_cast<const uint32_t*>(&r);
            }
            *reinterpret_cast<uint4*>(y) = make_uint4(out[0], out[1], out[2], out[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float4 b = reinterpret_cast<const float4*>(base)[i];
                b.x += o[4 * i], b.y += o[4 * i + 1], b.z += o[4 * i + 2], b.w += o[4 * i + 3];
                reinterpret_cast<float4*>(y)[i] = b;
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i < left) {
            const float v = as_float(base[i]) + o[i];
            if constexpr (sizeof(T) == 2) y[i] = __float2half_rn(v);
            else y[i] = v;
        }
    }
}

template <int kRankTiles, typename T>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 2) lora_kernel(const Params p) {
    constexpr bool kTwo = sizeof(T) == 4;                    // two fp16 numbers for a value of the vectors
    using L = Layout<kRankTiles>;
    extern __shared__ float4 shared[];
    float* sums = reinterpret_cast<float*>(shared);          // [warp][16 kRankTiles][kTokPad]; then the vectors [rank][kTokPad]
    float* part = sums + L::sums(p.rank);                    // [rank][kTokPad], read by the whole cluster
    float* largest = part + L::part(p.rank);                 // [warp][kTok], [kTok]
    __half* hi = reinterpret_cast<__half*>(largest + (kWarps + 1) * kTok);   // [kTok][row]
    const int row = L::row(p.rank);
    __half* lo = hi + kTok * row;

    dev::programmatic_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int cta = blockIdx.x % kCluster, z = blockIdx.x / kCluster % p.per_tile;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x / kCluster / p.per_tile) * kTok;

    // the tile's adapters, in the order of their first tokens; -1: tokens without one, which take base as it is
    const bool there = n0 + lane < p.N;
    int mine = there ? p.adapter[n0 + lane] : -2;
    if (there && (mine < 0 || mine >= p.count)) mine = -1;
    const unsigned same = __match_any_sync(0xFFFFFFFFu, mine);
    const bool first = lane == __ffs(same) - 1 && (mine >= 0 || (mine == -1 && p.base != p.Y));
    const unsigned groups = __ballot_sync(0xFFFFFFFFu, first);
    const int G = __popc(groups);
    if (G == 0) return;
    // more clusters than adapters: they share an adapter's output rows; else a cluster takes several adapters in turn
    const int sharers = p.per_tile > G ? (p.per_tile - z % G + G - 1) / G : 1, share = p.per_tile > G ? z / G : 0;
    const int step = p.per_tile > G ? G : p.per_tile;
    const int blocks = (p.M + kOut - 1) / kOut;
    if (share * kBlocksOfCluster >= blocks) return;

    for (int d = z % step; d < G; d += p.per_tile) {
        const int lead = __fns(groups, 0, d + 1);
        const int a = __shfl_sync(0xFFFFFFFFu, mine, lead);
        const unsigned members = __shfl_sync(0xFFFFFFFFu, same, lead);
        const int block0 = (share * kCluster + cta) * kWarps + w;
        if (a < 0) {
            constexpr int kPieces = kOut * sizeof(T) / 16;   // 16-byte pieces of a token's block
            for (int b = block0; b < blocks; b += sharers * kBlocksOfCluster) {
                const int m0 = b * kOut;
                const bool whole = p.wide_y && m0 + kOut <= p.M;
                for (int t = whole ? lane / kPieces : 0; t < kTok; t += whole ? 32 / kPieces : 1) {
                    if (!(members >> t & 1)) continue;
                    const T* from = static_cast<const T*>(p.base) + (n0 + t) * p.ldbase + m0;
                    T* to = static_cast<T*>(p.Y) + (n0 + t) * p.ldy + m0;
                    if (whole) {
                        reinterpret_cast<uint4*>(to)[lane % kPieces] = reinterpret_cast<const uint4*>(from)[lane % kPieces];
                    } else {
                        for (int i = lane; i < kOut && m0 + i < p.M; i += 32) to[i] = from[i];
                    }
                }
            }
            continue;
        }
        int rank = p.ranks != nullptr ? p.ranks[a] : p.rank;
        rank = rank < 0 ? 0 : rank > p.rank ? p.rank : rank;
        const int prank = padded_rank(rank);

        // A x over this CTA's eighth of K
        const __half* A = p.A + a * p.stride_a;
        const int steps = (p.K + 31) / 32;
        const int s0 = static_cast<int>(static_cast<int64_t>(steps) * cta / kCluster), s1 = static_cast<int>(static_cast<int64_t>(steps) * (cta + 1) / kCluster);
        for (int r0 = 0; r0 < rank; r0 += 16 * kRankTiles) {
            float acc[kRankTiles][4][4] = {};
            for (int s = s0 + w; s < s1; s += kWarps) {
                const int k = s * 32 + 8 * c;
                uint4 x[4], v[kRankTiles][2];
#pragma unroll
                for (int i = 0; i < kRankTiles; ++i) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = r0 + 16 * i + 8 * h + g;
                        v[i][h] = r < rank ? dev::load8(A + r * p.lda, k, p.K, p.wide_a) : make_uint4(0, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    x[t] = members >> (8 * t + g) & 1 ? dev::load8(p.X + (n0 + 8 * t + g) * p.ldx, k, p.K, p.wide_x) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (!(members >> (8 * t) & 0xFFu)) continue;
#pragma unroll
                    for (int i = 0; i < kRankTiles; ++i) {
                        dev::mma_f16(acc[i][t], v[i][0].x, v[i][1].x, v[i][0].y, v[i][1].y, x[t].x, x[t].y);
                        dev::mma_f16(acc[i][t], v[i][0].z, v[i][1].z, v[i][0].w, v[i][1].w, x[t].z, x[t].w);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kRankTiles; ++i) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    float* at = sums + (w * 16 * kRankTiles + 16 * i + g) * kTokPad + 8 * t + 2 * c;
                    *reinterpret_cast<float2*>(at) = make_float2(acc[i][t][0], acc[i][t][1]);
                    *reinterpret_cast<float2*>(at + 8 * kTokPad) = make_float2(acc[i][t][2], acc[i][t][3]);
                }
            }
            __syncthreads();
            for (int r = w; r < 16 * kRankTiles && r0 + r < rank; r += kWarps) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) sum += sums[(i * 16 * kRankTiles + r) * kTokPad + lane];
                part[(r0 + r) * kTokPad + lane] = sum;
            }
            __syncthreads();
        }
        cluster.sync();

        // the whole sums, scaled; the largest of a token decides its power of two
        const float scale = p.scales != nullptr ? p.scales[a] : 1.0f;
        float top = 0.0f;
        for (int r = w; r < prank; r += kWarps) {
            float sum = 0.0f;
            if (r < rank) {
#pragma unroll
                for (int i = 0; i < kCluster; ++i) sum += cluster.map_shared_rank(part, i)[r * kTokPad + lane];
            }
            sum *= scale;
            sums[r * kTokPad + lane] = sum;
            top = fmaxf(top, fabsf(sum));
        }
        largest[w * kTok + lane] = top;
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");    // this CTA has read the others' sums
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWarps; ++i) top = fmaxf(top, largest[i * kTok + lane]);
        // 2^14 <= top * up < 2^15 (values that are tiny, infinite or NaN keep a factor that is a plain number)
        const int exponent = max(27, min(254, __float_as_int(top) >> 23 & 255));
        const float up = __int_as_float((127 + 127 + 14 - exponent) << 23);
        if (w == 0) largest[kWarps * kTok + lane] = __int_as_float((exponent - 14) << 23);
        for (int r = w; r < prank; r += kWarps) {
            const float v = sums[r * kTokPad + lane] * up;
            const __half h = __float2half_rn(v);
            hi[lane * row + r] = h;
            if constexpr (kTwo) lo[lane * row + r] = __float2half_rn(v - __half2float(h));
        }
        __syncthreads();

        // B t, added to base
        const __half* B = p.B + a * p.stride_b;
        for (int b = block0; b < blocks; b += sharers * kBlocksOfCluster) {
            const int m0 = b * kOut + 8 * g;                 // a lane's eight consecutive output rows
            float acc[4][4][4] = {};
            for (int k0 = 0; k0 < rank; k0 += 32) {
                uint4 v[4][2];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i / 2][i % 2] = m0 + i < p.M ? dev::load8(B + (m0 + i) * p.ldb, k0 + 8 * c, rank, p.wide_b) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (!(members >> (8 * t) & 0xFFu)) continue;
                    const uint4 x = *reinterpret_cast<const uint4*>(hi + (8 * t + g) * row + k0 + 8 * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        dev::mma_f16(acc[t][i], v[i][0].x, v[i][1].x, v[i][0].y, v[i][1].y, x.x, x.y);
                        dev::mma_f16(acc[t][i], v[i][0].z, v[i][1].z, v[i][0].w, v[i][1].w, x.z, x.w);
                    }
                    if constexpr (kTwo) {
                        const uint4 y = *reinterpret_cast<const uint4*>(lo + (8 * t + g) * row + k0 + 8 * c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            dev::mma_f16(acc[t][i], v[i][0].x, v[i][1].x, v[i][0].y, v[i][1].y, y.x, y.y);
                            dev::mma_f16(acc[t][i], v[i][0].z, v[i][1].z, v[i][0].w, v[i][1].w, y.z, y.w);
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int n = 8 * t + 2 * c + h;
                    if (!(members >> n & 1) || m0 >= p.M) continue;
                    const float down = largest[kWarps * kTok + n];
                    float o[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[2 * i] = acc[t][i][h] * down, o[2 * i + 1] = acc[t][i][2 + h] * down;
                    add_store(static_cast<const T*>(p.base) + (n0 + n) * p.ldbase + m0, static_cast<T*>(p.Y) + (n0 + n) * p.ldy + m0, o, p.M - m0, p.wide_y);
                }
            }
        }
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // nobody reads this CTA's sums any more
    }
}

template <int kRankTiles, typename T>
spdp_status launch_form(const Params& p, int grid, cudaStream_t s) {
    SPDP_CUDA_TRY(launch_programmatic(lora_kernel<kRankTiles, T>, dim3(static_cast<unsigned>(grid)), kThreads, Layout<kRankTiles>::bytes(p.rank, sizeof(T) == 4), s, p));
    return SPDP_OK;
}

template <int kRankTiles>
spdp_status configure_form(int rank) {
    SPDP_CUDA_TRY(cudaFuncSetAttribute(lora_kernel<kRankTiles, __half>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(Layout<kRankTiles>::bytes(rank, false))));
    SPDP_CUDA_TRY(cudaFuncSetAttribute(lora_kernel<kRankTiles, float>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(Layout<kRankTiles>::bytes(rank, true))));
    return SPDP_OK;
}

}  // namespace

spdp_status current_device(int* device, int* sms) {
    static std::mutex mu;
    static int known[64] = {};
    SPDP_CUDA_TRY(cudaGetDevice(device));
    if (*device < 0 || *device >= 64) return SPDP_ERR_UNSUPPORTED_SHAPE;
    std::lock_guard<std::mutex> lock(mu);
    if (known[*device] == 0) SPDP_CUDA_TRY(cudaDeviceGetAttribute(&known[*device], cudaDevAttrMultiProcessorCount, *device));
    *sms = known[*device];
    return SPDP_OK;
}

static spdp_status configure_lora_kernel(int device) {
    static std::mutex mu;
    static bool configured[64] = {};
    std::lock_guard<std::mutex> lock(mu);
    if (configured[device]) return SPDP_OK;
    spdp_status st = configure_form<1>(16);
    if (st == SPDP_OK) st = configure_form<2>(32);
    if (st == SPDP_OK) st = configure_form<4>(SPDP_MAX_RANK);
    configured[device] = st == SPDP_OK;
    return st;
}

spdp_status launch_lora(const LoraCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    spdp_status st = current_device(&device, &sms);
    if (st == SPDP_OK) st = configure_lora_kernel(device);
    if (st != SPDP_OK) return st;
    const int64_t size = call.ydt == SPDP_Y_F32 ? 4 : 2;
    Params p = {};
    p.X = call.X, p.adapter = call.adapter, p.A = call.A, p.B = call.B, p.ranks = call.ranks, p.scales = call.scales, p.base = call.base, p.Y = call.Y;
    p.ldx = call.ldx, p.lda = call.lda, p.stride_a = call.stride_a, p.ldb = call.ldb, p.stride_b = call.stride_b, p.ldbase = call.ldbase, p.ldy = call.ldy;
    p.N = static_cast<int>(call.N), p.K = static_cast<int>(call.K), p.M = static_cast<int>(call.M);
    p.count = static_cast<int>(call.count), p.rank = call.rank;
    p.wide_x = rows_aligned16(call.X, call.ldx, 2);
    p.wide_a = rows_aligned16(call.A, call.lda | call.stride_a, 2);
    p.wide_b = rows_aligned16(call.B, call.ldb | call.stride_b, 2);
    p.wide_y = rows_aligned16(call.base, call.ldbase, size) && rows_aligned16(call.Y, call.ldy, size);
    // Clusters of a tile: enough for two CTAs per SM, no more than there is work for
    const int tiles = (p.N + kTok - 1) / kTok, blocks = (p.M + kOut - 1) / kOut;
    const int64_t most = static_cast<int64_t>(p.N < kTok ? p.N : kTok) * ((blocks + kBlocksOfCluster - 1) / kBlocksOfCluster);
    int64_t per_tile = 2 * sms / kCluster / tiles;
    if (per_tile > most) per_tile = most;
    if (per_tile < 1) per_tile = 1;
    p.per_tile = static_cast<int>(per_tile);
    const int grid = static_cast<int>(tiles * per_tile * kCluster);
    if (call.ydt == SPDP_Y_F32)
        return p.rank <= 16 ? launch_form<1, float>(p, grid, s) : p.rank <= 32 ? launch_form<2, float>(p, grid, s) : launch_form<4, float>(p, grid, s);
    return p.rank <= 16 ? launch_form<1, __half>(p, grid, s) : p.rank <= 32 ? launch_form<2, __half>(p, grid, s) : launch_form<4, __half>(p, grid, s);
}

}  // namespace spdp
