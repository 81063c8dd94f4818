// Low-rank adapters of many requests beside a shared projection: y_n = base_n + s_a B_a (A_a x_n), where a is the adapter of
// token n.  Folding B A into a statically pruned W would fill its zeros, so an adapter of a packed layer has to stay beside it.
//
// The work is the bytes: x, base and y once, the weights of the adapters in use; the products are a few times the rank per byte.
// Both products run on mma.sync with tokens as the 8 columns and weight rows as the 16 rows, fragments loaded straight from
// memory: a lane holds 8 consecutive elements of a row, the same on both sides.
//
// Tokens are brought together by adapter, 256 of them (a window) at a time, into tiles of up to 32 (8 where the tokens are few)
// that share one: the plan of a window, laid out on the device.
//
// First product: a cluster of 8 CTAs to a tile, or to as many tiles as bring all of them into one round; each of a tile's CTAs
// multiplies its share of K (its warps split that again), and the partial sums meet through distributed shared memory in a fixed
// order.  The vectors between the products are kept in fp16 for the second one, scaled per token by a power of two (so that neither
// end of the range is lost): one rounding of 2^-11 on a term that is added to a 16-bit result; for 32-bit results a second fp16
// number holds what the first one lost.
//
// Second product, a kernel of its own: the blocks of 64 output rows of all tiles stand in one line that is dealt out evenly to the
// warps, base comes to shared memory one block ahead.  For up to 16 tokens one launch does both products: the clusters keep
// the vectors and go on to the output rows.
//
// 1024 tokens of 28672 x 8192, rank 16, 16-bit results: 42 us of which the first kernel takes 13 and the second 28 (base and Y at 4.2
// TB/s); the first is bound by its chain (plan, two rounds of loads, exchange of the sums), the second by the waits between the
// steps of a block at the 11 warps that its registers allow.  8 tokens of rank 64: two such chains, 13.7 us where the 28 MB are in L2 (the
// same call again), 17 to 21 where they are not.
#include <cooperative_groups.h>

#include <mutex>

#include "mma_f16.cuh"
#include "spdp_internal.h"

namespace cg = cooperative_groups;

namespace spdp {
namespace {

constexpr int kMostCols = 4;        // column blocks of 8 tokens in a tile: 1 or 4
constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kCluster = 8;
constexpr int kExpandWarps = 4;     // of a CTA of the second kernel
constexpr int kOut = 64;            // output rows of a warp's block
constexpr int kBlocksOfCluster = kCluster * kWarps;
// Up to here one launch does both products, though clusters that share a tile all compute its vectors (us, one launch against two: 8
// tokens of rank 16, 4096 x 4096, 6.4 : 8.7; 16 of rank 64, 28672 x 8192, 15.7 : 20.0, of rank 256 53 : 61; 32 of rank 16, 11008 x 4096,
// 13.0 : 11.3).
constexpr int kFusedTokens = 16;
// Up to here tiles of the first product are 8 tokens, which loads further ahead; beyond, 32 that read A once (4 adapters of rank 16:
// 512 tokens of 8192 x 28672 equal, 1024 39 against 41 us; 8 of rank 64, 500 tokens of 8192 x 8192 27 against 30, 128 18 : 24).
constexpr int kFewTokens = 512;

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
    int per_window;                 // clusters (first or only kernel), CTAs (second) of a window, among which its work is dealt out
    bool wide_y;                    // base and Y: rows of whole 16-byte pieces, on such boundaries
    // what the first kernel leaves for the second: [N][padded rank] fp16, for 32-bit results twice, and a factor to each token
    __half* vectors;
    float* factors;
    struct Plan* plans;             // of the windows, for the second kernel
};

int64_t between(int64_t v, int64_t low, int64_t high) { return v > high ? high : v < low ? low : v; }

__host__ __device__ inline int padded_rank(int rank) { return (rank + 31) & ~31; }

// Shared memory of the first product, in floats.  Rows of kTok + 8 floats: the fragments' stores meet no bank twice.
template <int kRankTiles, int kCols>
struct Layout {
    static constexpr int kTok = 8 * kCols, kPad = kTok + 8;
    static __host__ __device__ int sums(int rank) {
        const int warps = kWarps * 16 * kRankTiles, all = padded_rank(rank);
        return (warps > all ? warps : all) * kPad;
    }
    static __host__ __device__ int part(int rank) { return padded_rank(rank) * kPad; }
    static __host__ __device__ int row(int rank) { return padded_rank(rank) + 8; }       // halves of a token's vector
    static __host__ __device__ size_t bytes(int rank, bool two) {
        return 4u * (sums(rank) + part(rank) + (kWarps + 1) * 32) + 2u * kTok * row(rank) * (two ? 2 : 1);
    }
};

// The tokens of a request stand together, those of an adapter need not: 256 consecutive tokens, a window, are brought together by
// adapter, and a tile is up to kTok tokens of a window that share one.  So 256 tokens that draw from 15 adapters are 15 to 23
// tiles of 32, not 8 tiles of 13 adapters each.
constexpr int kWindow = kThreads;
struct Tile {
    int adapter;                    // -1: none
    unsigned bits;                  // first place in `order`, 9 bits; tokens, 6 bits; rank
    __device__ __forceinline__ int first() const { return bits & 511; }
    __device__ __forceinline__ int count() const { return bits >> 9 & 63; }
    __device__ __forceinline__ int rank() const { return bits >> 15; }
};
__device__ __forceinline__ Tile make_tile(int adapter, int first, int count, int rank) {
    return {adapter, static_cast<unsigned>(first | count << 9 | rank << 15)};
}
struct __align__(128) Plan {
    int tiles;
    unsigned char order[kWindow];   // the window's tokens, by adapter
    Tile tile[kWindow];
};

__device__ __forceinline__ int rank_of(const Params& p, int a) {
    const int rank = p.ranks != nullptr ? p.ranks[a] : p.rank;
    return rank < 0 ? 0 : rank > p.rank ? p.rank : rank;
}

// The plan of a window with tiles of `tok` tokens, into shared memory (all threads; ends with a barrier); `wide`, if not null, gets
// the plan with tiles of 32.  Tokens without an adapter take base as it is: in place they are left out, and in `plan` unless it is
// for both products (kBare).
template <bool kBare>
__device__ void make_plan(const Params& p, int64_t n0, int tok, Plan& plan, Plan* wide) {
    __shared__ int2 entries[kWarps][32];                        // of each warp: an adapter, its tokens and (2^8) the first one's lane
    __shared__ int starts[kWindow], warp_sums[kWarps], warp_entries[kWarps];
    const int t = threadIdx.x, lane = t & 31, w = t >> 5, tokens = p.N - n0 < kWindow ? static_cast<int>(p.N - n0) : kWindow;
    int mine = t < tokens ? p.adapter[n0 + t] : -2;
    if (t < tokens && (mine < 0 || mine >= p.count)) mine = p.base != p.Y ? -1 : -2;
    const int rank = mine >= 0 ? rank_of(p, mine) : 0;
    const unsigned same = __match_any_sync(0xFFFFFFFFu, mine), below = (1u << lane) - 1u;
    const int leader = __ffs(same) - 1;
    const unsigned leaders = __ballot_sync(0xFFFFFFFFu, lane == leader);
    if (lane == leader) entries[w][__popc(leaders & below)] = make_int2(mine, __popc(same) | lane << 8);
    if (lane == 0) warp_entries[w] = __popc(leaders);
    __syncthreads();
    int all = 0, before = 0, lead = kWindow;                    // tokens that share the adapter, those in front, the first of them
    for (int i = 0; i < kWarps && 32 * i < tokens; ++i) {
        for (int j = 0, n = warp_entries[i]; j < n; ++j) {
            const int2 e = entries[i][j];
            if (e.x != mine) continue;
            all += e.y & 255;
            if (i < w) before += e.y & 255;
            lead = min(lead, 32 * i + (e.y >> 8));
        }
    }
    before += __popc(same & below);
    const bool leads = mine != -2 && lead == t;
    // places, tiles and tiles of 32 of the adapters in front, ten bits each
    const int here = kBare || mine >= 0 ? all : 0;
    int sum = leads ? all | (here + tok - 1) / tok << 10 | (all + 31) / 32 << 20 : 0;
    const int own = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 31) warp_sums[w] = sum;
    __syncthreads();
    int front = 0, total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        if (i < w) front += warp_sums[i];
        total += warp_sums[i];
    }
    front += sum - own;
    const int start = front & 1023;
    if (leads) {
        starts[t] = start;
        for (int i = 0, at = front >> 10 & 1023; i * tok < here; ++i) plan.tile[at + i] = make_tile(mine, start + i * tok, min(tok, all - i * tok), rank);
        if (wide != nullptr)
            for (int i = 0, at = front >> 20; 32 * i < all; ++i) wide->tile[at + i] = make_tile(mine, start + 32 * i, min(32, all - 32 * i), rank);
    }
    __syncthreads();
    if (mine != -2) plan.order[starts[lead] + before] = static_cast<unsigned char>(t);
    if (t == 0) plan.tiles = total >> 10 & 1023;
    __syncthreads();
    if (wide != nullptr) {
        wide->order[t] = plan.order[t];
        if (t == 0) wide->tiles = total >> 20;
    }
}

// A warp's block of output: 64 rows, eight to a lane (for two tokens of each column block).  kWide: base and Y are read and
// written 16 bytes at a time, and a lane's rows are neighbours, 8 g + e; else value by value, and the rows are 8 e + g, so that
// the lanes' are.
template <bool kWide>
__device__ __forceinline__ int row_of(int g, int e) { return kWide ? 8 * g + e : 8 * e + g; }

template <typename T>
__device__ __forceinline__ T sum_of(T base, float add) {
    if constexpr (sizeof(T) == 2) return __float2half_rn(__half2float(base) + add);
    else return base + add;
}
// Eight neighbours of Y: base's, at `from` (16-byte aligned, as `to` is), plus f o.
template <typename T>
__device__ __forceinline__ void add_eight(T* to, const T* from, const float (&o)[8], float f) {
    union { uint4 bits[sizeof(T) / 2]; T v[8]; } x;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) x.bits[i] = reinterpret_cast<const uint4*>(from)[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = sum_of(x.v[i], o[i] * f);
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4*>(to)[i] = x.bits[i];
}

// The second product for a warp's block of output rows from m_block on, added to base, for the `count` tokens n0 + list[..].
// `hi`, `lo`: vectors, `row` halves apart, and `factors` that undo their scaling, by place in the list or (kByToken) by token.
// `old`: base's block in shared memory, [place][kOldRow], or null: it is read where it is.  a < 0: base as it is.
template <typename T>
constexpr int kOldRow = kOut + 16 / static_cast<int>(sizeof(T));     // a token's values of a block, and 16 bytes

template <typename T, int kCols, int kAlign, bool kWide, bool kByToken>
__device__ __forceinline__ void expand_block(const Params& p, int64_t n0, const unsigned char* list, int count, int a, int rank, int m_block, const __half* hi,
                                             const __half* lo, int row, const float* factors, const T* old) {
    constexpr bool kTwo = sizeof(T) == 4;
    constexpr int kStep = kCols < 2 || (kAlign == 16 && kWide) ? kCols : 2;     // column blocks at a time
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int left = p.M - m_block;                              // rows of the block that exist
    const bool there = row_of<kWide>(g, 0) < left;               // kWide: M is a multiple of 8, so all eight or none
    uint4 v[4][2], x[kCols];
    const __half* B = p.B + a * p.stride_b + (m_block + row_of<kWide>(g, 0)) * p.ldb;
    const int64_t apart = (kWide ? 1 : 8) * p.ldb;
    auto weights = [&](int k0) {
        const __half* at = B;
#pragma unroll
        for (int i = 0; i < 8; ++i, at += apart) v[i / 2][i % 2] = dev::load8<kAlign>(at, k0 + 8 * c, row_of<kWide>(g, i) < left ? rank : 0);
        if (kAlign == 16 && rank % 8 != 0) {                     // what stands behind an adapter's own rank
#pragma unroll
            for (int i = 0; i < 8; ++i) dev::cut8(v[i / 2][i % 2], k0 + 8 * c, rank);
        }
    };
    int token[kCols][2], place[kCols];                           // of the lane's columns 2 c and 2 c + 1; the vector of its column g
#pragma unroll
    for (int t = 0; t < kCols; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) token[t][h] = 8 * t + 2 * c + h < count ? list[8 * t + 2 * c + h] : -1;
        place[t] = 8 * t + g >= count ? -1 : kByToken ? list[8 * t + g] : 8 * t + g;
    }
    auto vectors = [&](int k0) {
#pragma unroll
        for (int t = 0; t < kCols; ++t) {
            x[t] = make_uint4(0, 0, 0, 0);
            if (place[t] >= 0) x[t] = *reinterpret_cast<const uint4*>(hi + place[t] * row + k0 + 8 * c);
        }
    };
    float down[kCols][2];
    if (a >= 0) {
        if (rank > 0) weights(0), vectors(0);
#pragma unroll
        for (int t = 0; t < kCols; ++t) {
#pragma unroll
            for (int h = 0; h < 2; ++h) down[t][h] = token[t][h] >= 0 ? factors[kByToken ? token[t][h] : 8 * t + 2 * c + h] : 0.0f;
        }
    }
    const T* base = static_cast<const T*>(p.base) + n0 * p.ldbase + m_block;
    T* y = static_cast<T*>(p.Y) + n0 * p.ldy + m_block;
#pragma unroll
    for (int t0 = 0; t0 < kCols; t0 += kStep) {
        if (8 * t0 >= count) break;
        float acc[kStep][4][4] = {};
        if (a >= 0) {
            for (int k0 = 0; k0 < rank; k0 += 32) {
                if (rank > 32 && (k0 > 0 || t0 > 0)) weights(k0), vectors(k0);
#pragma unroll
                for (int t = 0; t < kStep; ++t) {
                    uint4 z = make_uint4(0, 0, 0, 0);
                    if (kTwo && place[t0 + t] >= 0) z = *reinterpret_cast<const uint4*>(lo + place[t0 + t] * row + k0 + 8 * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        dev::mma_f16(acc[t][i], v[i][0].x, v[i][1].x, v[i][0].y, v[i][1].y, x[t0 + t].x, x[t0 + t].y);
                        dev::mma_f16(acc[t][i], v[i][0].z, v[i][1].z, v[i][0].w, v[i][1].w, x[t0 + t].z, x[t0 + t].w);
                    }
                    if constexpr (kTwo) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            dev::mma_f16(acc[t][i], v[i][0].x, v[i][1].x, v[i][0].y, v[i][1].y, z.x, z.y);
                            dev::mma_f16(acc[t][i], v[i][0].z, v[i][1].z, v[i][0].w, v[i][1].w, z.z, z.w);
                        }
                    }
                }
            }
        }
        if constexpr (kWide) {
#pragma unroll
            for (int t = 0; t < kStep; ++t) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int n = token[t0 + t][h];
                    if (!there || n < 0) continue;
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = acc[t][e / 2][2 * (e % 2) + h];
                    T* to = y + n * p.ldy + 8 * g;
                    const T* from = old != nullptr ? old + (8 * (t0 + t) + 2 * c + h) * kOldRow<T> + 8 * g : base + n * p.ldbase + 8 * g;
                    if (a < 0) {
#pragma unroll
                        for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(from)[i];
                    } else {
                        add_eight(to, from, o, down[t0 + t][h]);
                    }
                }
            }
        } else {                                                 // all values of base first: a store ends what may be read ahead of it
            T in[kStep][2][8];
#pragma unroll
            for (int e = 0; e < 16 * kStep; ++e) {
                const int t = e / 16, h = e / 8 % 2, n = token[t0 + t][h];
                if (n >= 0 && row_of<kWide>(g, e % 8) < left) in[t][h][e % 8] = base[n * p.ldbase + row_of<kWide>(g, e % 8)];
            }
#pragma unroll
            for (int e = 0; e < 16 * kStep; ++e) {
                const int t = e / 16, h = e / 8 % 2, n = token[t0 + t][h];
                if (n < 0 || row_of<kWide>(g, e % 8) >= left) continue;
                const T b = in[t][h][e % 8];
                y[n * p.ldy + row_of<kWide>(g, e % 8)] = a < 0 ? b : sum_of(b, acc[t][e % 8 / 2][2 * (e % 2) + h] * down[t0 + t][h]);
            }
        }
    }
}

// kSplit: this kernel ends with the vectors, in memory; else it does the second product too.
template <int kRankTiles, int kCols, typename T, bool kSplit, int kAlign>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 2) lora_kernel(const Params p) {
    constexpr bool kTwo = sizeof(T) == 4;                    // two fp16 numbers for a value of the vectors
    // steps of 32 k whose loads are on their way at once; a step takes 4 kCols + 8 kRankTiles registers
    constexpr int kBatch = kCols == 1 ? (kRankTiles == 4 ? 2 : 4) : kRankTiles == 1 ? 2 : 1;
    using L = Layout<kRankTiles, kCols>;
    constexpr int kTok = L::kTok, kPad = L::kPad;
    extern __shared__ float4 shared[];
    float* sums = reinterpret_cast<float*>(shared);          // [warp][16 kRankTiles][kPad]; then the vectors [rank][kPad]
    float* part = sums + L::sums(p.rank);                    // [rank][kPad], read by the whole cluster
    float* largest = part + L::part(p.rank);                 // [warp][32], factors [32]
    float* factors = largest + kWarps * 32;
    __half* hi = reinterpret_cast<__half*>(factors + 32);    // [kTok][row]
    const int row = L::row(p.rank);
    __half* lo = hi + kTok * row;

    dev::programmatic_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int cta = blockIdx.x % kCluster, z = blockIdx.x / kCluster % p.per_window;
    const int64_t window = blockIdx.x / kCluster / p.per_window, n0 = window * kWindow;
    __shared__ Plan plan;
    make_plan<!kSplit>(p, n0, kTok, plan, kSplit && cta == 0 && z == 0 ? p.plans + window : nullptr);
    const int tiles = plan.tiles;
    if (tiles == 0) return;
    // more clusters than tiles: they share a tile's output rows; else a cluster takes several tiles in turn
    const bool more = !kSplit && p.per_window > tiles;
    const int sharers = more ? (p.per_window - z % tiles + tiles - 1) / tiles : 1, share = more ? z / tiles : 0;
    const int blocks = (p.M + kOut - 1) / kOut;
    if (share * kBlocksOfCluster >= blocks) return;
    // kSplit: where there are more tiles than clusters, a cluster takes 2, 4 or 8 at a time, with fewer CTAs to each (256 tokens with
    // adapters of their own, rank 16, 4096 x 11008: 64 -> 51 us; 2048 that share 8: 38.7 -> 34.3)
    static_assert(kCluster == 8, "CTAs of a tile: 1 << shift");
    int shift = 3;
    if constexpr (kSplit)
        while (shift > 0 && tiles > p.per_window << (3 - shift)) --shift;
    const int sharing = 1 << shift, at_once = kCluster >> shift, mate = cta & (sharing - 1);

    for (int d0 = more ? z % tiles : z * at_once; d0 < tiles; d0 += p.per_window * at_once) {
        const int d = d0 + (cta >> shift);
        const Tile tile = d < tiles ? plan.tile[d] : make_tile(-1, 0, 0, 0);
        const int a = tile.adapter, count = tile.count(), rank = tile.rank(), prank = padded_rank(rank);
        const unsigned char* list = plan.order + tile.first();
        const int block0 = (share * kCluster + cta) * kWarps + w;
        if (!kSplit && a < 0) {                              // the same for the whole cluster
            for (int b = block0; b < blocks; b += sharers * kBlocksOfCluster)
                expand_block<T, kCols, kAlign, true, false>(p, n0, list, count, a, 0, b * kOut, hi, lo, row, factors, nullptr);
            continue;
        }

        // A x over this CTA's share of K (a < 0: its rank is 0, and it only keeps step with the cluster)
        const __half* A = p.A + a * p.stride_a;
        int token[kCols];                                    // the lane's, behind n0
#pragma unroll
        for (int t = 0; t < kCols; ++t) token[t] = 8 * t + g < count ? list[8 * t + g] : -1;
        const __half* X = p.X + n0 * p.ldx;
        const int steps = (p.K + 31) / 32;
        const int s0 = steps * mate >> shift, s1 = steps * (mate + 1) >> shift;
        for (int r0 = 0; r0 < rank; r0 += 16 * kRankTiles) {
            float acc[kRankTiles][kCols][4] = {};
            for (int s = s0 + w; s < s1; s += kBatch * kWarps) {
                uint4 x[kBatch][kCols], v[kBatch][kRankTiles][2];
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    const int k = s + j * kWarps < s1 ? (s + j * kWarps) * 32 + 8 * c : p.K;
                    const __half* at = A + (r0 + g) * p.lda;
#pragma unroll
                    for (int i = 0; i < 2 * kRankTiles; ++i, at += 8 * p.lda) v[j][i / 2][i % 2] = dev::load8<kAlign>(at, k, r0 + 8 * i + g < rank ? p.K : 0);
#pragma unroll
                    for (int t = 0; t < kCols; ++t) x[j][t] = dev::load8<kAlign>(X + token[t] * p.ldx, k, token[t] >= 0 ? p.K : 0);
                }
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
#pragma unroll
                    for (int t = 0; t < kCols; ++t) {
                        if (8 * t >= count) continue;
#pragma unroll
                        for (int i = 0; i < kRankTiles; ++i) {
                            dev::mma_f16(acc[i][t], v[j][i][0].x, v[j][i][1].x, v[j][i][0].y, v[j][i][1].y, x[j][t].x, x[j][t].y);
                            dev::mma_f16(acc[i][t], v[j][i][0].z, v[j][i][1].z, v[j][i][0].w, v[j][i][1].w, x[j][t].z, x[j][t].w);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kRankTiles; ++i) {
#pragma unroll
                for (int t = 0; t < kCols; ++t) {
                    float* at = sums + (w * 16 * kRankTiles + 16 * i + g) * kPad + 8 * t + 2 * c;
                    *reinterpret_cast<float2*>(at) = make_float2(acc[i][t][0], acc[i][t][1]);
                    *reinterpret_cast<float2*>(at + 8 * kPad) = make_float2(acc[i][t][2], acc[i][t][3]);
                }
            }
            __syncthreads();
            for (int e = threadIdx.x; e < 16 * kRankTiles * kTok; e += kThreads) {
                const int r = e / kTok, n = e % kTok;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) sum += sums[(i * 16 * kRankTiles + r) * kPad + n];
                if (r0 + r < rank) part[(r0 + r) * kPad + n] = sum;
            }
            __syncthreads();
        }
        cluster.sync();

        // the whole sums, scaled; the largest of a token decides its power of two
        constexpr int kRows = kThreads / kTok;               // ranks at a time; a thread keeps its token
        const int n = threadIdx.x % kTok, r_first = threadIdx.x / kTok;
        const float scale = p.scales != nullptr && a >= 0 ? p.scales[a] : 1.0f;
        float top = 0.0f;
        for (int r = r_first; r < prank; r += kRows) {
            float sum = 0.0f;
            if (r < rank) {
                if (sharing == kCluster) {
#pragma unroll
                    for (int i = 0; i < kCluster; ++i) sum += cluster.map_shared_rank(part, i)[r * kPad + n];
                } else {
                    for (int i = cta - mate; i < cta - mate + sharing; ++i) sum += cluster.map_shared_rank(part, i)[r * kPad + n];
                }
            }
            sum *= scale;
            sums[r * kPad + n] = sum;
            top = fmaxf(top, fabsf(sum));
        }
#pragma unroll
        for (int i = kTok; i < 32; i *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, i));
        if (lane < kTok) largest[w * 32 + lane] = top;
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");    // this CTA has read the others' sums
        __syncthreads();
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) top = fmaxf(top, largest[i * 32 + n]);
        // 2^14 <= top * up < 2^15 (values that are tiny, infinite or NaN keep a factor that is a plain number)
        const int exponent = max(27, min(254, __float_as_int(top) >> 23 & 255));
        const float up = __int_as_float((127 + 127 + 14 - exponent) << 23);
        if (threadIdx.x < kTok) factors[n] = __int_as_float((exponent - 14) << 23);
        for (int r = r_first; r < prank; r += kRows) {
            const float v = sums[r * kPad + n] * up;
            const __half h = __float2half_rn(v);
            hi[n * row + r] = h;
            if constexpr (kTwo) lo[n * row + r] = __float2half_rn(isinf(v) ? 0.0f : v - __half2float(h));      // Inf loses nothing
        }
        __syncthreads();

        if constexpr (kSplit) {
            // each of the tile's CTAs writes as many of its vectors
            const int width = padded_rank(p.rank), pieces = prank / 8, mine = kTok >> shift;
            const int64_t all = static_cast<int64_t>(p.N) * width;
            for (int e = threadIdx.x; e < mine * pieces; e += kThreads) {
                const int t = mate * mine + e / pieces, k = e % pieces * 8;
                if (t >= count) continue;
                __half* to = p.vectors + (n0 + list[t]) * width + k;
                *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(hi + t * row + k);
                if constexpr (kTwo) *reinterpret_cast<uint4*>(to + all) = *reinterpret_cast<const uint4*>(lo + t * row + k);
            }
            const int t = mate * mine + threadIdx.x;
            if (threadIdx.x < mine && t < count) p.factors[n0 + list[t]] = factors[t];
        } else {
            for (int b = block0; b < blocks; b += sharers * kBlocksOfCluster)
                expand_block<T, kCols, kAlign, true, false>(p, n0, list, count, a, rank, b * kOut, hi, lo, row, factors, nullptr);
        }
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // nobody reads this CTA's sums any more
    }
}

// What its registers are cut for (at 4 the forms for odd rows spill: 500 tokens, rank 20, 4001 x 4098, 30.5 us against 20.8).
constexpr int kExpandCtasOfSm = 3;

// The second product where it has a kernel of its own.  The blocks of all tiles of a window stand in one line, an equal run of
// them to each warp of the window's CTAs, however many tiles there are.  A warp copies base of the next block to shared
// memory while it works on one (kWide; else base is read where it is).  kShort: 16-byte loads and ranks up to 32, the usual case;
// a tile's vectors stay in registers for all its blocks, and the weights of the next block are on their way too.
template <typename T, int kAlign, bool kWide, bool kShort>
__global__ void __launch_bounds__(32 * kExpandWarps, kExpandCtasOfSm) lora_expand_kernel(const Params p) {
    constexpr int kTok = 8 * kMostCols, kPiece = 16 / sizeof(T), kPieces = kOut / kPiece;        // values of 16 bytes, such pieces of a row
    extern __shared__ float4 shared[];
    dev::programmatic_start();
    const int blocks = (p.M + kOut - 1) / kOut, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t window = blockIdx.x / p.per_window, n0 = window * kWindow;
    const int me = blockIdx.x % p.per_window * kExpandWarps + w, warps = p.per_window * kExpandWarps, width = padded_rank(p.rank);
    const Plan* plan = p.plans + window;
    const unsigned units = static_cast<unsigned>(plan->tiles) * static_cast<unsigned>(blocks), each = units / warps, more = units % warps;
    unsigned u = me * each + min(static_cast<unsigned>(me), more);
    const unsigned end = u + each + (me < static_cast<int>(more) ? 1 : 0);
    if (u >= end) return;
    T* olds = reinterpret_cast<T*>(shared) + w * 2 * kTok * kOldRow<T>;          // two blocks
    auto copy = [&](Tile tile, int b, int to) {
        if constexpr (kWide) {
            const unsigned char* list = plan->order + tile.first();
            const int count = tile.count();
            const T* from = static_cast<const T*>(p.base) + n0 * p.ldbase + b * kOut;
            const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(olds + to * kTok * kOldRow<T>));
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int n = i * (32 / kPieces) + lane / kPieces, part = lane % kPieces;
                if (n < count && b * kOut + part * kPiece < p.M)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + (n * kOldRow<T> + part * kPiece) * static_cast<int>(sizeof(T))),
                                 "l"(from + list[n] * p.ldbase + part * kPiece) : "memory");
            }
        }
    };
    int b = static_cast<int>(u % blocks), d = static_cast<int>(u / blocks);
    Tile tile = plan->tile[d];
    copy(tile, b, 0);
    if constexpr (kWide) asm volatile("cp.async.commit_group;" ::: "memory");
    int rank = tile.rank();
    const __half* hi = p.vectors + n0 * width;
    if constexpr (kShort) {
        constexpr bool kTwo = sizeof(T) == 4;
        const int g = lane >> 2, c = lane & 3;
        const __half* lo = hi + static_cast<int64_t>(p.N) * width;
        int token[kMostCols][2];                                 // of the lane's columns
        float down[kMostCols][2];
        uint4 x[kMostCols], z[kTwo ? kMostCols : 1], v[4][2], ahead[4][2];
        auto enter = [&]() {                                     // a tile
            const unsigned char* list = plan->order + tile.first();
            const int count = tile.count();
#pragma unroll
            for (int t = 0; t < kMostCols; ++t) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    token[t][h] = 8 * t + 2 * c + h < count ? list[8 * t + 2 * c + h] : -1;
                    down[t][h] = token[t][h] >= 0 && tile.adapter >= 0 ? p.factors[n0 + token[t][h]] : 0.0f;
                }
                x[t] = make_uint4(0, 0, 0, 0);
                if constexpr (kTwo) z[t] = make_uint4(0, 0, 0, 0);
                if (8 * t + g < count && 8 * c < rank) {
                    const int at = list[8 * t + g] * width + 8 * c;
                    x[t] = *reinterpret_cast<const uint4*>(hi + at);
                    if constexpr (kTwo) z[t] = *reinterpret_cast<const uint4*>(lo + at);
                }
            }
        };
        auto weights = [&](uint4 (&into)[4][2], int adapter, int its_rank, int block) {
            const int m0 = block * kOut + 8 * g;
            const __half* at = p.B + adapter * p.stride_b + m0 * p.ldb;
#pragma unroll
            for (int j = 0; j < 8; ++j, at += p.ldb) into[j / 2][j % 2] = dev::load8<16>(at, 8 * c, m0 < p.M ? its_rank : 0);
        };
        enter();
        weights(v, tile.adapter, rank, b);
        for (int i = 0; u < end; ++u, i ^= 1) {
            const bool last = b + 1 == blocks;                   // of its tile
            Tile next = tile;
            if (u + 1 < end) {
                if (last) next = plan->tile[d + 1];
                copy(next, last ? 0 : b + 1, i ^ 1);
                weights(ahead, next.adapter, next.rank(), last ? 0 : b + 1);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
            if (rank % 8 != 0) {                                 // what stands behind an adapter's own rank
#pragma unroll
                for (int j = 0; j < 8; ++j) dev::cut8(v[j / 2][j % 2], 8 * c, rank);
            }
            const T* old = olds + i * kTok * kOldRow<T> + 8 * g;
            T* y = static_cast<T*>(p.Y) + n0 * p.ldy + b * kOut + 8 * g;
            const bool there = b * kOut + 8 * g < p.M;
#pragma unroll
            for (int t = 0; t < kMostCols; ++t) {
                if (8 * t >= tile.count()) break;
                float acc[4][4] = {};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dev::mma_f16(acc[j], v[j][0].x, v[j][1].x, v[j][0].y, v[j][1].y, x[t].x, x[t].y);
                    if constexpr (kTwo) dev::mma_f16(acc[j], v[j][0].x, v[j][1].x, v[j][0].y, v[j][1].y, z[t].x, z[t].y);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dev::mma_f16(acc[j], v[j][0].z, v[j][1].z, v[j][0].w, v[j][1].w, x[t].z, x[t].w);
                    if constexpr (kTwo) dev::mma_f16(acc[j], v[j][0].z, v[j][1].z, v[j][0].w, v[j][1].w, z[t].z, z[t].w);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!there || token[t][h] < 0) continue;
                    const T* from = old + (8 * t + 2 * c + h) * kOldRow<T>;
                    T* to = y + token[t][h] * p.ldy;
                    if (tile.adapter < 0) {
#pragma unroll
                        for (int j = 0; j < static_cast<int>(sizeof(T)) / 2; ++j) reinterpret_cast<uint4*>(to)[j] = reinterpret_cast<const uint4*>(from)[j];
                    } else {
                        float o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = acc[e / 2][2 * (e % 2) + h];
                        add_eight(to, from, o, down[t][h]);
                    }
                }
            }
            __syncwarp();                                        // all lanes have read the block before it is overwritten
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j / 2][j % 2] = ahead[j / 2][j % 2];
            if (last) {
                tile = next, rank = next.rank(), ++d, b = 0;
                if (u + 1 < end) enter();
            } else {
                ++b;
            }
        }
    } else {
        for (int i = 0; u < end; ++u, i ^= 1) {
            const bool last = b + 1 == blocks;                       // of its tile
            Tile next = tile;
            if (u + 1 < end) {
                if (last) next = plan->tile[d + 1];
                copy(next, last ? 0 : b + 1, i ^ 1);
            }
            if constexpr (kWide) {
                asm volatile("cp.async.commit_group;" ::: "memory");
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncwarp();
            }
            expand_block<T, kMostCols, kAlign, kWide, true>(p, n0, plan->order + tile.first(), tile.count(), tile.adapter, rank, b * kOut, hi,
                                                            hi + static_cast<int64_t>(p.N) * width, width, p.factors + n0, kWide ? olds + i * kTok * kOldRow<T> : nullptr);
            if constexpr (kWide) __syncwarp();                       // all lanes have read the block before it is overwritten
            if (last) {
                tile = next, ++d, b = 0;
                rank = tile.rank();
            } else {
                ++b;
            }
        }
    }
}

template <typename T, int kAlign, bool kWide, bool kShort>
cudaError_t launch_expand(Params p, int device, int sms, cudaStream_t s) {
    static std::mutex mu;
    static bool configured[64] = {};
    const size_t bytes = kWide ? kExpandWarps * 2 * 8 * kMostCols * kOldRow<T> * sizeof(T) : 0;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[device]) {
            const cudaError_t e = cudaFuncSetAttribute(lora_expand_kernel<T, kAlign, kWide, kShort>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
            if (e != cudaSuccess) return e;
        }
        configured[device] = true;
    }
    // as many CTAs as the GPU holds at once, no more than there can be blocks
    const int64_t windows = (p.N + kWindow - 1) / kWindow, blocks = (p.M + kOut - 1) / kOut, slots = kExpandCtasOfSm * static_cast<int64_t>(sms);
    p.per_window = static_cast<int>(between((slots + windows - 1) / windows, 1, ((p.N < kWindow ? p.N : kWindow) * blocks + kExpandWarps - 1) / kExpandWarps));
    const int64_t size = windows * p.per_window;
    if (size > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_programmatic(lora_expand_kernel<T, kAlign, kWide, kShort>, dim3(static_cast<unsigned>(size)), 32 * kExpandWarps, bytes, s, p);
}

template <int kRankTiles, int kCols, typename T, bool kSplit, int kAlign>
spdp_status launch_form(const Params& p, int windows, int device, cudaStream_t s) {
    static std::mutex mu;
    static bool configured[64] = {};
    constexpr int kMostRank = kRankTiles == 4 ? SPDP_MAX_RANK : 16 * kRankTiles;
    using L = Layout<kRankTiles, kCols>;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[device])
            SPDP_CUDA_TRY(cudaFuncSetAttribute(lora_kernel<kRankTiles, kCols, T, kSplit, kAlign>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(L::bytes(kMostRank, sizeof(T) == 4))));
        configured[device] = true;
    }
    const dim3 grid(static_cast<unsigned>(windows) * static_cast<unsigned>(p.per_window) * kCluster);
    SPDP_CUDA_TRY(launch_programmatic(lora_kernel<kRankTiles, kCols, T, kSplit, kAlign>, grid, kThreads, L::bytes(p.rank, sizeof(T) == 4), s, p));
    return SPDP_OK;
}

template <int kCols, typename T, bool kSplit, int kAlign>
spdp_status launch_rank(const Params& p, int windows, int device, cudaStream_t s) {
    if (p.rank <= 16) return launch_form<1, kCols, T, kSplit, kAlign>(p, windows, device, s);
    if (p.rank <= 32) return launch_form<2, kCols, T, kSplit, kAlign>(p, windows, device, s);
    return launch_form<4, kCols, T, kSplit, kAlign>(p, windows, device, s);
}

template <typename T>
spdp_status launch_typed(Params p, int align, int device, int sms, cudaStream_t s) {
    const int blocks = (p.M + kOut - 1) / kOut, cluster_slots = 2 * sms / kCluster;
    if (p.N <= kFusedTokens && align == 16 && p.wide_y) {
        // Clusters of a tile: two CTAs per SM in all, no more than there is work for
        const int64_t most = static_cast<int64_t>(p.N) * ((blocks + kBlocksOfCluster - 1) / kBlocksOfCluster);
        p.per_window = static_cast<int>(between(cluster_slots, 1, most));
        return launch_rank<1, T, false, 16>(p, 1, device, s);
    }
    const bool few = p.N <= kFewTokens;
    const int windows = (p.N + kWindow - 1) / kWindow, width = padded_rank(p.rank);
    const size_t vectors = (2ull * p.N * width * (sizeof(T) == 4 ? 2 : 1) + 127) / 128 * 128, factors = (4ull * p.N + 127) / 128 * 128;
    void* scratch = nullptr;
    spdp_status st = scratch_alloc(device, vectors + factors + windows * sizeof(Plan), s, &scratch);
    if (st != SPDP_OK) return st;
    p.vectors = static_cast<__half*>(scratch);
    p.factors = reinterpret_cast<float*>(static_cast<char*>(scratch) + vectors);
    p.plans = reinterpret_cast<Plan*>(static_cast<char*>(scratch) + vectors + factors);
    p.per_window = static_cast<int>(between(cluster_slots / windows, 1, p.N < kWindow ? p.N : kWindow));
    if (align == 16) st = few ? launch_rank<1, T, true, 16>(p, windows, device, s) : launch_rank<kMostCols, T, true, 16>(p, windows, device, s);
    else if (few) st = align == 4 ? launch_rank<1, T, true, 4>(p, windows, device, s) : launch_rank<1, T, true, 2>(p, windows, device, s);
    else st = align == 4 ? launch_rank<kMostCols, T, true, 4>(p, windows, device, s) : launch_rank<kMostCols, T, true, 2>(p, windows, device, s);
    if (st == SPDP_OK) {
        const cudaError_t e = align == 16 && p.wide_y && p.rank <= 32 ? launch_expand<T, 16, true, true>(p, device, sms, s)
                              : align == 16 ? (p.wide_y ? launch_expand<T, 16, true, false>(p, device, sms, s) : launch_expand<T, 16, false, false>(p, device, sms, s))
                              : align == 4  ? (p.wide_y ? launch_expand<T, 4, true, false>(p, device, sms, s) : launch_expand<T, 4, false, false>(p, device, sms, s))
                                            : (p.wide_y ? launch_expand<T, 2, true, false>(p, device, sms, s) : launch_expand<T, 2, false, false>(p, device, sms, s));
        if (e != cudaSuccess) {
            note_cuda_error(e, "lora_expand_kernel");
            st = SPDP_ERR_CUDA;
        }
    }
    SPDP_CUDA_TRY(cudaFreeAsync(scratch, s));
    return st;
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

spdp_status launch_lora(const LoraCall& call, cudaStream_t s) {
    int device = 0, sms = 0;
    const spdp_status st = current_device(&device, &sms);
    if (st != SPDP_OK) return st;
    const int64_t size = call.ydt == SPDP_Y_F32 ? 4 : 2;
    Params p = {};
    p.X = call.X, p.adapter = call.adapter, p.A = call.A, p.B = call.B, p.ranks = call.ranks, p.scales = call.scales, p.base = call.base, p.Y = call.Y;
    p.ldx = call.ldx, p.lda = call.lda, p.stride_a = call.stride_a, p.ldb = call.ldb, p.stride_b = call.stride_b, p.ldbase = call.ldbase, p.ldy = call.ldy;
    p.N = static_cast<int>(call.N), p.K = static_cast<int>(call.K), p.M = static_cast<int>(call.M);
    p.count = static_cast<int>(call.count), p.rank = call.rank;
    p.wide_y = call.M % 8 == 0 && rows_aligned16(call.base, call.ldbase, size) && rows_aligned16(call.Y, call.ldy, size);
    // 16-byte loads where every row of X, A and B starts on such a boundary and has whole pieces; else 4-byte or 2-byte ones
    int align = 16;
    for (const int v : {rows_alignment(call.X, call.ldx, 2), rows_alignment(call.A, call.lda | call.stride_a, 2), rows_alignment(call.B, call.ldb | call.stride_b, 2)})
        if (v < align) align = v;
    align = align == 16 && call.K % 8 == 0 && call.rank % 8 == 0 ? 16 : align >= 4 ? 4 : 2;
    return call.ydt == SPDP_Y_F32 ? launch_typed<float>(p, align, device, sms, s) : launch_typed<__half>(p, align, device, sms, s);
}

}  // namespace spdp
