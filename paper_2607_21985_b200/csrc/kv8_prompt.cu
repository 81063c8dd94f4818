// Attention over the 8-bit cache for requests with many new tokens: prompts and pieces of them, on the 5th-generation tensor cores.
//
// The rows of a key head, token by token its query heads, are cut into blocks of kTiles tiles of 128 rows; a block's keys, 128 to
// a unit, are those that any of its tokens sees.  The units of all blocks and heads stand in one line that is cut into equal
// runs, one to a CTA (kv8.cuh); a first small kernel writes down where each block begins.
//
// Inside a CTA: a warp goes through the run and tells the others its pieces of blocks, two bring rows of q to shared memory, a warpgroup
// turns codes into fp16 operand tiles there, a thread issues the products, and a warpgroup to each tile has the softmax, a row to a
// thread.  Scores are Q K^T into tensor memory; weights go back there, over the scores, as the
// first operand of the product with the values, whose sums stay in tensor memory through the block.  While one tile's scores become
// weights the tensor cores work on the other's.  Codes times their scale are fp16 numbers, so both operands of the first product and
// the values of the second are exact; the weights are rounded to fp16 (2^-11, the one rounding besides the result's).
// What bounds it: the way of a tile's scores, from the products through the softmax (some 1900 cycles a unit, 1024 of them the exponentials of
// a scheduler's 32 rows) and back, two tiles side by side: 3700 cycles a unit of 256 rows, whose products are 2048; and the power limit, at 1.89
// GHz.  4096 tokens of 64 and 8 heads of 128: 305 to 326 us by itself, 0.9 PFLOP/s (327 to 347 with the store of its keys and values).  Under a cap 520 while a warp's
// scores are within a quarter of it; where they are not, 1470 to 1540 (an exponential and a quotient more to a score; 2045 tokens of 32 and 8 heads in pieces with a
// window 118, 174 and 412).  Tried and not kept:
// units of 64 keys with scores for two of them (384 us), a pair of CTAs to 512 rows (cta_group::2, 327 us against 330, with 512 rows to a block), a
// thread to each tile's products (382 to 410), two threads to a row (359), turns at the exponentials (340 to 381), part of them by a polynomial (376
// and up), the softmax as two short loops over a row (332, but capped ones 209 against 185), code of its own for each softmax warpgroup (its code
// then leaves the instruction cache: 45 % slower).
//
// The order of a unit's keys is what suits the operand tiles, and the same in both: row n of the keys' tile is token 2 (n % 64 / 16) + n % 2 +
// 8 (n % 4 / 2) of cell 4 (n / 64) + 2 (n / 8 % 2) + n / 4 % 2.  So the 8 keys of a 16-byte piece of a dimension's row of the values' tile are
// words of two cells that one lane has, and the lanes' pieces of either tile fall into different banks.
#include <cfloat>
#include <mutex>

#include "kv8.cuh"

namespace spdp {
namespace {

using namespace kv8;

constexpr int kUnitCells = 8, kUnitKeys = kUnitCells * kCell;
constexpr int kTileRows = 128;
constexpr int kThreads = 512;           // warps 0-3 and 4-7: softmax; 8-11: codes to operands; 12: products; 13: pieces; 14, 15: rows of q
constexpr int kRowBytes = 128;          // of an operand tile: 64 fp16 numbers, in the 128-byte swizzle
constexpr int kAtomBytes = 8 * kRowBytes;
constexpr int kShortList = 192, kShortRequests = 32;     // up to so many blocks of so many requests each CTA lists itself, which saves a kernel (333 tokens of 12 and 3 heads: 24.5 -> 22.5 us)
constexpr int kFlags = 8;               // units whose cells' existence is kept
constexpr float kHeadroom = 8.0f, kSlack = 6.5f;       // weights are below 2^(kHeadroom + kSlack); 12 and 2.5 scale the sums anew more often: 336 -> 342 us
template <int kDim>
struct Form {
    static constexpr int kTiles = kDim == 256 ? 1 : 2;
    static constexpr int kStages = kDim == 256 ? 1 : 2;                 // of the keys' and of the values' tiles
    static constexpr int kRows = kTiles * kTileRows;
    static constexpr int kKeyBytes = kUnitKeys * kDim * 2, kQueryBytes = kTileRows * kDim * 2;
    static constexpr int kSums = 256;                                   // first tensor-memory column of the sums; scores of tile t at 128 t
    // Registers of a thread by its warpgroup (the second softmax warpgroup has nothing to do where there is one tile: the codes' gets them); with the
    // 128 of the launch the four come to the same sum.
    static constexpr int kSoftmaxRegs = 176, kSecondRegs = kTiles == 2 ? kSoftmaxRegs : 40, kDecodeRegs = kTiles == 2 ? 112 : 232, kOtherRegs = kTiles == 2 ? 48 : 64;
    static_assert(kSoftmaxRegs + kSecondRegs + kDecodeRegs + kOtherRegs == 4 * 128, "the launch's registers");
    static constexpr int kOperands = kTiles * kQueryBytes + 2 * kStages * kKeyBytes;
};

struct alignas(16) Block {              // of rows, and the cells with keys that any of its tokens sees, as one line (kv8.cuh, Request)
    int start, length;                  // in the line of one head
    int request, row0, rows;
    int n0, before, keys;               // the request's first token, its keys before that, all its keys
    int sink_cells, low_cell, cells;
    int earliest, latest;               // positions of the block's tokens
    int pad[3];
    __device__ __forceinline__ int cell_at(int i) const { return i < sink_cells ? i : i - sink_cells + low_cell; }
};
struct PromptParams {
    AttnParams a;
    Block* blocks;
    int* totals;                        // blocks; length of the line of one head; null: each CTA lists the blocks itself
    int most_list;                      // blocks that there can be
    bool negative;                      // the scale; a.scale is its size
    bool wide16;                        // rows of y on 16-byte boundaries
    uint32_t magic, shift;              // of a division by the group
    // n / group for 0 <= n < 2^31: with 2^shift >= group, magic = (2^shift - group) 2^32 / group, rounded down, plus 1 (Granlund and Montgomery)
    __device__ __forceinline__ int by_group(int n) const { return static_cast<int>((__umulhi(magic, static_cast<uint32_t>(n)) + static_cast<uint32_t>(n)) >> shift); }
};

template <int kRows>
__device__ __forceinline__ Block block_of(const AttnParams& p, int b, int row0) {
    const Request rq = request_of(p, b);
    Block s = {};
    s.request = b, s.row0 = row0, s.rows = min(kRows, rq.n * p.group - row0), s.n0 = rq.n0, s.before = rq.length - rq.n, s.keys = rq.length;
    s.earliest = s.before + row0 / p.group, s.latest = s.before + (row0 + s.rows - 1) / p.group;
    if (p.window > 0) {
        s.low_cell = max(max(s.earliest, 0) + 1 - p.window, 0) / kCell;
        s.sink_cells = min((p.sinks + kCell - 1) / kCell, s.low_cell);
    }
    s.cells = s.sink_cells + max(s.latest, 0) / kCell + 1 - s.low_cell;         // one at least
    s.length = triple_length((s.cells + kUnitCells - 1) / kUnitCells);
    return s;
}

// ---- where each block begins

constexpr int kListThreads = 1024;

__device__ __forceinline__ int scan_add(int mine, int* sums, int* total) {       // the sum of the threads before this one; all threads, ends with a barrier
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int up_to = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, up_to, d);
        if (lane >= d) up_to += v;
    }
    if (lane == 31) sums[w] = up_to;
    __syncthreads();
    if (w == 0) {
        const int all = sums[lane];
        int s = all;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, s, d);
            if (lane >= d) s += v;
        }
        __syncwarp();
        sums[lane] = s - all;
        if (lane == 31) sums[32] = s;
    }
    __syncthreads();
    const int r = sums[w] + up_to - mine;
    *total = sums[32];
    __syncthreads();
    return r;
}

template <int kRows>
__global__ void __launch_bounds__(kListThreads) kv8_blocks_kernel(const PromptParams p) {
    __shared__ int first[4096 + 1], sums[33];
    dev::programmatic_start();
    int total = 0;
    for (int base = 0; base < p.a.B; base += kListThreads) {    // the first block of each request
        const int b = base + threadIdx.x;
        int mine = 0, all;
        if (b < p.a.B) {
            const Request rq = request_of(p.a, b);
            mine = rq.cells > 0 ? (rq.n * p.a.group + kRows - 1) / kRows : 0;
        }
        const int at = total + scan_add(mine, sums, &all);
        if (b < p.a.B) first[b] = at;
        total += all;
    }
    __syncthreads();
    total = min(total, p.most_list);
    int length = 0;
    for (int base = 0; base < total; base += kListThreads) {
        const int i = base + threadIdx.x;
        int all;
        Block block = {};
        if (i < total) {
            const int b = request_at(first, p.a.B, i);
            block = block_of<kRows>(p.a, b, (i - first[b]) * kRows);
        }
        block.start = length + scan_add(block.length, sums, &all);
        if (i < total) p.blocks[i] = block;
        length += all;
    }
    if (threadIdx.x == 0) p.totals[0] = total, p.totals[1] = length;
}

// ---- a CTA's pieces of blocks, in order

struct alignas(16) Piece {
    Block block;
    int index, h;                       // the block's number, the key head
    int off, count;                     // units; count 0: no piece any more
    int whole, slot, last_cta;
    unsigned unit0;                     // units of the CTA before it
};
constexpr int kPieces = 4;              // that are known at a time

// ---- tensor cores, barriers

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// Shared-memory operand descriptor of tcgen05.mma, K-major rows of 128 bytes in the 128-byte swizzle: start address (in 16 bytes) in the lower
// half; in the upper the distance of 8 rows, the descriptor's version, the layout.
constexpr uint32_t kDescHigh = (kAtomBytes >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (1u << 16); }
// fp16 x fp16 -> fp32, both K-major, 128 rows, n columns
__device__ __forceinline__ constexpr uint32_t instr_desc(int n) { return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(kTileRows >> 4) << 24); }
__device__ __forceinline__ void mma_smem(uint32_t d, uint32_t a_low, uint32_t b_low, uint32_t id, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d), "r"(a_low), "r"(b_low), "r"(id), "r"(accumulate), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b_low, uint32_t id, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n mov.b64 b, {%2, %5};\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b_low), "r"(id), "r"(accumulate), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    unsigned e;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e != 0u;
}
__device__ __forceinline__ void barrier_init(uint64_t* bar, uint32_t arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }
constexpr int kWaitTries = 1 << 22;     // a wait that runs out (none should) ends its role: the rows of the piece that is worked on become NaN, later ones stay unwritten
constexpr int kDrainTries = 1 << 18;
__device__ __forceinline__ bool wait_parity(uint64_t* bar, unsigned parity, int limit = kWaitTries) {
    const uint32_t a = smem_u32(bar);
    for (int tries = 0; tries < limit; ++tries) {
        unsigned done;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(a), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

#define SPDP_R8(a, i) "=f"((a)[i]), "=f"((a)[i + 1]), "=f"((a)[i + 2]), "=f"((a)[i + 3]), "=f"((a)[i + 4]), "=f"((a)[i + 5]), "=f"((a)[i + 6]), "=f"((a)[i + 7])
#define SPDP_W8(a, i) "r"((a)[i]), "r"((a)[i + 1]), "r"((a)[i + 2]), "r"((a)[i + 3]), "r"((a)[i + 4]), "r"((a)[i + 5]), "r"((a)[i + 6]), "r"((a)[i + 7])
// 32 columns of tensor memory, the thread's lane.
__device__ __forceinline__ void tmem_load(uint32_t at, float* v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
                 "%28, %29, %30, %31}, [%32];"
                 : SPDP_R8(v, 0), SPDP_R8(v, 8), SPDP_R8(v, 16), SPDP_R8(v, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
                 "%28, %29, %30, %31, %32};" ::"r"(at), SPDP_W8(v, 0), SPDP_W8(v, 8), SPDP_W8(v, 16), SPDP_W8(v, 24) : "memory");
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Pairs of 32-bit numbers in one operation.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n fma.rn.f32x2 x, x, y, z;\n mov.b64 {%0, %1}, x;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 twice(float a) { return make_float2(a, a); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// The lowest n bits of 16: none below 0, all from 16 on.
__device__ __forceinline__ uint32_t low_bits(int n) { return (1u << min(max(n, 0), kCell)) - 1u; }

struct Barriers {
    uint64_t q_full[2], q_free[2], s_full[2], p_full[2][2], o_full[2], k_full[2], k_free[2], v_full[2], v_free[2], piece_full[kPieces], piece_free[kPieces], drained;
    uint32_t tmem;
    Piece pieces[kPieces];
    Block blocks[kShortList];           // where each CTA lists them
    alignas(16) int there[kFlags][4];   // of the units' cells, two bits to a decoding warp
};

// Key of column n of a unit, from the first key of its cell
__host__ __device__ constexpr int cell_of(int n) { return 4 * (n / 64) + 2 * (n / 8 % 2) + n / 4 % 2; }
__host__ __device__ constexpr int token_of(int n) { return 2 * (n % 64 / 16) + n % 2 + 8 * (n % 4 / 2); }

// The next piece for a role (whole warps, or one thread): null at the end, or where it does not come.
__device__ __forceinline__ const Piece* piece_at(Barriers* bars, unsigned i) {
    if (!wait_parity(&bars->piece_full[i % kPieces], (i / kPieces) & 1u)) return nullptr;
    const Piece* s = &bars->pieces[i % kPieces];
    return s->count > 0 ? s : nullptr;
}

// ---- pieces (a warp)

// The list of blocks into this CTA's shared memory, and the first CTA's also to where the join looks: (blocks, length of the line of one head).
template <int kRows>
__device__ __forceinline__ int2 list_blocks(const PromptParams& p, Barriers* bars) {
    const int lane = threadIdx.x & 31;
    int count = 0;                                              // of the lane's request
    if (lane < p.a.B) {
        const Request rq = request_of(p.a, lane);
        if (rq.cells > 0) count = (rq.n * p.a.group + kRows - 1) / kRows;
    }
    int up_to = count;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, up_to, d);
        if (lane >= d) up_to += v;
    }
    const int total = min(__shfl_sync(0xFFFFFFFFu, up_to, 31), p.most_list);
    int length = 0;
    for (int base = 0; base < total; base += 32) {
        const int i = base + lane;
        int b = 0;                                              // the first request whose blocks go on behind i
#pragma unroll
        for (int d = 16; d > 0; d /= 2)
            if (__shfl_sync(0xFFFFFFFFu, up_to, b + d - 1) <= i) b += d;
        b = min(b, p.a.B - 1);
        const int first = __shfl_sync(0xFFFFFFFFu, up_to - count, b);
        Block block = {};
        if (i < total) block = block_of<kRows>(p.a, b, (i - first) * kRows);
        int at = block.length;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, at, d);
            if (lane >= d) at += v;
        }
        block.start = length + at - block.length;
        length += __shfl_sync(0xFFFFFFFFu, at, 31);
        if (i < total) {
            bars->blocks[i] = block;
            if (blockIdx.x == 0) p.blocks[i] = block;
        }
    }
    __syncwarp();
    return make_int2(total, length);
}

template <int kRows>
__device__ __forceinline__ void piece_role(const PromptParams& p, Barriers* bars) {
    const int2 list = p.totals != nullptr ? make_int2(p.totals[0], p.totals[1]) : list_blocks<kRows>(p, bars);
    const Block* const blocks = p.totals != nullptr ? p.blocks : bars->blocks;
    const int lane = threadIdx.x & 31, n = list.x, length = list.y, total = length * p.a.heads, ctas = min(static_cast<int>(gridDim.x), total);
    int u = 0, stop = 0, index = 0, h = 0;
    if (static_cast<int>(blockIdx.x) < ctas) {
        u = run_start(total, ctas, blockIdx.x), stop = run_start(total, ctas, blockIdx.x + 1);
        h = u / length;
        const int v = u % length;
        for (int count = n; count > 1;) {                       // the last of the blocks index .. index + count - 1 that does not begin behind v
            const int step = (count + 31) / 32, last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, lane * step < count && blocks[index + lane * step].start <= v));
            const int end = index + count;
            index += last * step, count = min(step, end - index);
        }
    }
    unsigned i = 0, units = 0;
    for (bool more = true; more;) {
        Piece s;
        s.count = 0;
        while (u < stop && s.count <= 0) {
            s.block = blocks[index];
            const int start = h * length + s.block.start;
            s.off = max(0, u - start - kStart), s.count = max(0, min(s.block.length, stop - start) - kStart) - s.off;
            s.index = index, s.h = h, s.whole = s.count == s.block.length - kStart;
            s.slot = 2 * blockIdx.x + (i > 0 ? 1 : 0);          // what is not whole is the first piece of a run or the last
            s.last_cta = static_cast<int>(((static_cast<int64_t>(start) + s.block.length) * ctas - 1) / total);
            u = min(start + s.block.length, stop);
            if (++index == n) index = 0, ++h;                   // count <= 0: the run ends before the block's first unit
        }
        s.count = max(s.count, 0);
        s.unit0 = units, units += s.count;
        more = s.count > 0;
        if (i >= kPieces && !__all_sync(0xFFFFFFFFu, wait_parity(&bars->piece_free[i % kPieces], (i / kPieces - 1u) & 1u))) return;
        if (lane == 0) {
            if (more && s.off == 0 && !s.whole) p.a.open[blockIdx.x] = make_int4(s.index, s.h, s.slot, s.last_cta);     // the CTAs with the rest follow this one
            bars->pieces[i % kPieces] = s;
            arrive(&bars->piece_full[i % kPieces]);
        }
        __syncwarp();
        ++i;
    }
}

// ---- rows of q (a warp to each tile, or two to one)

template <int kDim>
__device__ __forceinline__ void query_role(const PromptParams& p, Barriers* bars, uint32_t queries, int warp) {
    using F = Form<kDim>;
    constexpr int kOfRow = kDim / 8;    // 16-byte pieces of a row
    const int lane = threadIdx.x & 31, tile = F::kTiles == 2 ? warp : 0, first = F::kTiles == 2 ? 0 : 64 * warp, count = F::kTiles == 2 ? 128 : 64;
    const AttnParams& a = p.a;
    const uint32_t my_queries = queries + tile * F::kQueryBytes;
    unsigned mine = 0;
    for (unsigned i = 0;; ++i) {
        const Piece* s = piece_at(bars, i);
        if (__any_sync(0xFFFFFFFFu, s == nullptr)) return;
        const int rows = s->block.rows - tile * kTileRows, row0 = s->block.row0 + tile * kTileRows, n0 = s->block.n0, h = s->h;
        if (rows > 0) {
            if (mine > 0 && !__all_sync(0xFFFFFFFFu, wait_parity(&bars->q_free[tile], (mine - 1u) & 1u))) return;
            ++mine;
#pragma unroll 4
            for (int e = lane; e < count * kOfRow; e += 32) {
                const int r = first + e / kOfRow, piece = e % kOfRow, row = row0 + min(r, rows - 1), token = p.by_group(row);
                const __half* from = a.q + (n0 + token) * a.ldq + static_cast<int64_t>(h * a.group + row - token * a.group) * kDim + 8 * piece;
                const uint32_t to = my_queries + piece / 8 * (kTileRows * kRowBytes) + r * kRowBytes + ((piece % 8) ^ (r & 7)) * 16;
                if (a.wide_q) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(r < rows ? 16 : 0) : "memory");   // zeros behind the last row
                else {
                    const unsigned short* x = reinterpret_cast<const unsigned short*>(from);
                    uint32_t v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = r < rows ? x[2 * j] | static_cast<uint32_t>(x[2 * j + 1]) << 16 : 0u;
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_operands();
            __syncwarp();
            if (lane == 0) arrive(&bars->q_full[tile]);
        }
        __syncwarp();
        if (lane == 0) arrive(&bars->piece_free[i % kPieces]);
    }
}

// ---- codes to operands

template <int kDim>
__device__ __forceinline__ void decode_role(const PromptParams& p, Barriers* bars, uint32_t keys, uint32_t values) {
    using F = Form<kDim>;
    constexpr int kLoads = kDim / 32;   // 16-byte loads of a side of a cell
    const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) & 3, g = lane >> 2, c = lane & 3;
    const AttnParams& a = p.a;
    const int in_page = (1 << a.cells_shift) - 1;
    const int64_t page_bytes = (static_cast<int64_t>(a.heads) << a.cells_shift) * cell_bytes(kDim);
    // places in the tiles: the lane's key g of a cell (the other one, g + 8, two rows on), 16 dimensions from 16 c; dimension g, 8 keys
    const uint32_t key_row = 16 * (g >> 1) + 8 * (w & 1) + 64 * (w >> 1) + (g & 1);
    const uint32_t value_at = g * kRowBytes + (((2 * c + (w & 1)) ^ g) << 4) + (w >> 1) * (kDim * kRowBytes);
    unsigned unit = 0;
    for (unsigned number = 0;; ++number) {
        const Piece* s = piece_at(bars, number);
        if (__any_sync(0xFFFFFFFFu, s == nullptr)) return;
        const Block& rq = s->block;
        const int count = s->count, line0 = s->off * kUnitCells + 2 * w;
        const int32_t* table = a.table + rq.request * a.table_stride;
        const unsigned char* head = a.cache + (static_cast<int64_t>(s->h) << a.cells_shift) * cell_bytes(kDim) + 16 * lane;
        auto place = [&](int i, int j) { return line0 + i * kUnitCells + j; };  // in the block's line, of cell j of the warp's in unit i
        auto pages_of = [&](int i) {                            // of the units i .. i + 15
            const int at = place(i + (lane >> 1), lane & 1);
            return i + (lane >> 1) < count && at < rq.cells ? table[rq.cell_at(at) >> a.cells_shift] : -1;
        };
        int pages = pages_of(0), pages_after = pages_of(16);
        uint4 k[2][kLoads], v[2][kLoads];
        float2 scale[2], scale_next[2];
        bool ok[2], ok_next[2];
        const unsigned char* from[2];
        auto locate = [&](int i) {
            if (i > 0 && (i & 15) == 0) pages = pages_after, pages_after = pages_of(i + 16);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const unsigned page = __shfl_sync(0xFFFFFFFFu, pages, (2 * i + j) & 31);
                ok_next[j] = i < count && page < a.pages;
                from[j] = head + static_cast<int64_t>(ok_next[j] ? page : 0u) * page_bytes + (rq.cell_at(place(i, j)) & in_page) * cell_bytes(kDim);
            }
        };
        auto load_keys = [&]() {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                scale_next[j] = make_float2(0.0f, 0.0f);
                if (ok_next[j]) scale_next[j] = *reinterpret_cast<const float2*>(from[j] + 2 * kCell * kDim - 16 * lane);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    k[j][i] = make_uint4(0, 0, 0, 0);
                    if (ok_next[j]) k[j][i] = *reinterpret_cast<const uint4*>(from[j] + 512 * i);
                }
            }
        };
        auto load_values = [&]() {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    v[j][i] = make_uint4(0, 0, 0, 0);
                    if (ok_next[j]) v[j][i] = *reinterpret_cast<const uint4*>(from[j] + kCell * kDim + 512 * i);
                }
            }
        };
        auto scaled = [](uint32_t codes, __half2 f) {
            const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&codes), f);
            return *reinterpret_cast<const uint32_t*>(&r);
        };
        auto put = [](uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t t) { asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(t) : "memory"); };
        locate(0);
        load_keys();
        load_values();
        for (int i = 0; i < count; ++i, ++unit) {
            const unsigned stage = unit % F::kStages, parity = (unit / F::kStages - 1u) & 1u;
            int key[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) scale[j] = scale_next[j], ok[j] = ok_next[j], key[j] = rq.cell_at(place(i, j)) * kCell;
            if (unit >= F::kStages && !__all_sync(0xFFFFFFFFu, wait_parity(&bars->k_free[stage], parity))) return;
            if (lane == 0) bars->there[unit % kFlags][w] = (ok[0] ? 1 : 0) | (ok[1] ? 2 : 0);
            const uint32_t k_tile = keys + stage * F::kKeyBytes;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const __half2 f = __float2half2_rn(scale[j].x);
#pragma unroll
                for (int t = 0; t < kLoads; ++t) {              // 64 dimensions t / 2, key g + 8 (t % 2)
                    const uint32_t row = key_row + 4 * j + 2 * (t & 1), at = k_tile + (t >> 1) * (kUnitKeys * kRowBytes) + row * kRowBytes;
                    const uint4& x = k[j][t];
                    put(at + (((2 * c) ^ (row & 7)) << 4), scaled(low_codes(x.x), f), scaled(high_codes(x.x), f), scaled(low_codes(x.y), f), scaled(high_codes(x.y), f));
                    put(at + (((2 * c + 1) ^ (row & 7)) << 4), scaled(low_codes(x.z), f), scaled(high_codes(x.z), f), scaled(low_codes(x.w), f), scaled(high_codes(x.w), f));
                }
            }
            fence_operands();
            __syncwarp();
            if (lane == 0) arrive(&bars->k_full[stage]);
            locate(i + 1);
            load_keys();
            if (unit >= F::kStages && !__all_sync(0xFFFFFFFFu, wait_parity(&bars->v_free[stage], parity))) return;
            if (max(key[0], key[1]) + kCell > rq.keys) {     // behind the last key: whatever the cell holds there
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t keep = 0;
#pragma unroll
                    for (int m = 0; m < 4; ++m) keep |= key[j] + 2 * c + (m & 1) + 8 * (m >> 1) < rq.keys ? 0xFFu << 8 * m : 0u;
#pragma unroll
                    for (int t = 0; t < kLoads; ++t) v[j][t].x &= keep, v[j][t].y &= keep, v[j][t].z &= keep, v[j][t].w &= keep;
                }
            }
            const uint32_t v_tile = values + stage * F::kKeyBytes + value_at;
            const __half2 f0 = __float2half2_rn(scale[0].y), f1 = __float2half2_rn(scale[1].y);
#pragma unroll
            for (int t = 0; t < kLoads; ++t) {                  // dimensions 32 t + 8 m + g
                const uint32_t x[4] = {v[0][t].x, v[0][t].y, v[0][t].z, v[0][t].w}, y[4] = {v[1][t].x, v[1][t].y, v[1][t].z, v[1][t].w};
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    put(v_tile + (32 * t + 8 * m) * kRowBytes, scaled(low_codes(x[m]), f0), scaled(high_codes(x[m]), f0), scaled(low_codes(y[m]), f1), scaled(high_codes(y[m]), f1));
            }
            fence_operands();
            __syncwarp();
            if (lane == 0) arrive(&bars->v_full[stage]);
            load_values();
        }
        __syncwarp();
        if (lane == 0) arrive(&bars->piece_free[number % kPieces]);
    }
}

// ---- products (one thread)

template <int kDim>
__device__ __forceinline__ void product_role(const PromptParams& p, Barriers* bars, uint32_t queries, uint32_t keys, uint32_t values, uint32_t tmem) {
    using F = Form<kDim>;
    const uint32_t q_low = desc_low(queries), k_low = desc_low(keys), v_low = desc_low(values);
    const uint32_t id_scores = instr_desc(kUnitKeys) | (p.negative ? 1u << 13 : 0u);    // the first operand times -1
    constexpr uint32_t kIdSums = instr_desc(kDim);
    unsigned piece_of[2] = {0, 0}, unit = 0, weights_of[2] = {0, 0};    // pieces and units so far, of each tile
    bool ok = true, issued = false;
    auto scores = [&](int t, unsigned u) {
        const uint32_t stage = u % F::kStages;
#pragma unroll
        for (int kk = 0; kk < kDim / 16; ++kk)
            mma_smem(tmem + 128 * t, q_low + ((t * F::kQueryBytes + kk / 4 * (kTileRows * kRowBytes) + kk % 4 * 32) >> 4),
                     k_low + ((stage * F::kKeyBytes + kk / 4 * (kUnitKeys * kRowBytes) + kk % 4 * 32) >> 4), id_scores, kk > 0);
        issued = true;
        commit(&bars->s_full[t]);
    };
    for (unsigned number = 0; ok; ++number) {
        const Piece* s = piece_at(bars, number);
        if (s == nullptr) break;
        const int tiles = F::kTiles == 2 && s->block.rows > kTileRows ? 2 : 1, count = s->count;
        arrive(&bars->piece_free[number % kPieces]);
        ok = wait_parity(&bars->k_full[unit % F::kStages], (unit / F::kStages) & 1u);
        for (int t = 0; ok && t < tiles; ++t) {
            ok = wait_parity(&bars->q_full[t], piece_of[t]++ & 1u);
            if (!ok) break;
            fence_after();
            scores(t, unit);
            if (count == 1) commit(&bars->q_free[t]);
        }
        if (ok) commit(&bars->k_free[unit % F::kStages]);
        for (int i = 0; ok && i < count; ++i, ++unit) {
            const uint32_t stage = unit % F::kStages;
            ok = wait_parity(&bars->v_full[stage], (unit / F::kStages) & 1u);
            for (int t = 0; ok && t < tiles; ++t) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ok = ok && wait_parity(&bars->p_full[t][half], weights_of[t] & 1u);
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int kk = 4 * half; kk < 4 * half + 4; ++kk)
                        mma_tmem(tmem + F::kSums + t * kDim, tmem + 128 * t + 8 * kk, v_low + ((stage * F::kKeyBytes + half * (kDim * kRowBytes) + kk % 4 * 32) >> 4), kIdSums,
                                 i > 0 || kk > 0);
                }
                if (!ok) break;
                ++weights_of[t];
                if (i + 1 < count) {
                    if (t == 0) ok = wait_parity(&bars->k_full[(unit + 1) % F::kStages], ((unit + 1) / F::kStages) & 1u);
                    if (!ok) break;
                    scores(t, unit + 1);
                    if (i + 2 == count) commit(&bars->q_free[t]);
                } else commit(&bars->o_full[t]);
            }
            if (!ok) break;
            commit(&bars->v_free[stage]);
            if (i + 1 < count) commit(&bars->k_free[(unit + 1) % F::kStages]);
        }
    }
    if (issued) {                       // tensor memory is not freed under running products
        commit(&bars->drained);
        wait_parity(&bars->drained, 0u, kDrainTries);
    }
}

// ---- softmax of a tile's rows, a row to a thread

template <int kDim, bool kCap>
__device__ __forceinline__ void softmax_role(const PromptParams& p, Barriers* bars, uint32_t tmem, int tile) {
    using F = Form<kDim>;
    const AttnParams& a = p.a;
    const int t = threadIdx.x & 127, lane = t & 31, w = t >> 5;
    const uint32_t lanes = static_cast<uint32_t>(32 * w) << 16, at_scores = tmem + 128 * tile + lanes, at_sums = tmem + F::kSums + tile * kDim + lanes;
    unsigned units = 0, pieces = 0;                             // of this tile
    bool ok = true;
    for (unsigned number = 0;; ++number) {
        const Piece* const s = piece_at(bars, number);
        if (__any_sync(0xFFFFFFFFu, s == nullptr)) return;
        const Block& block = s->block;
        const int rows = block.rows - tile * kTileRows;
        if (rows <= 0) {                                        // the block ends in the first tile
            __syncwarp();
            if (lane == 0) arrive(&bars->piece_free[number % kPieces]);
            continue;
        }
        const int row = block.row0 + tile * kTileRows + min(t, rows - 1), token = p.by_group(row), position = block.before + token, count = s->count;
        // The piece's units whose every key every token of the block sees (one run of them), if the pages exist.  (Found once, in registers: a load from
        // shared memory waits behind the exponentials of the scheduler's other warps.)
        const int off = s->off, past = a.window > 0 ? max(block.latest + 1 - a.window, 0) : 0;     // keys before `past` are behind some window
        const int whole_begin = (block.sink_cells + (past + kCell - 1) / kCell - block.low_cell + kUnitCells - 1) / kUnitCells - off;
        const int whole_end = (block.earliest < 0 ? 0 : block.sink_cells + (block.earliest + 1) / kCell - block.low_cell) / kUnitCells - off;
        const unsigned unit0 = s->unit0;
        float top = kLowest, weight = 0.0f;
        for (int i = 0; i < count; ++i, ++units) {
            ok = ok && __all_sync(0xFFFFFFFFu, wait_parity(&bars->s_full[tile], units & 1u));
            if (!ok) break;
            fence_after();
            float x[128];
#pragma unroll
            for (int j = 0; j < 4; ++j) tmem_load(at_scores + 32 * j, x + 32 * j);
            const int4 there = *reinterpret_cast<const int4*>(bars->there[(unit0 + i) % kFlags]);
            const bool whole = i >= whole_begin && i < whole_end && (there.x & there.y & there.z & there.w) == 3;
            tmem_loaded();
            if constexpr (kCap) {
                float most = 0.0f;
#pragma unroll
                for (int n = 0; n < 128; n += 4) most = fmaxf(most, fmaxf(fmaxf(fabsf(x[n]), fabsf(x[n + 1])), fmaxf(fabsf(x[n + 2]), fabsf(x[n + 3]))));
                if (__any_sync(0xFFFFFFFFu, !(most * a.scale <= a.cap_near))) {
#pragma unroll
                    for (int n = 0; n < 128; ++n) x[n] = capped(a, x[n] * a.scale);
                } else {                                        // as capped_near, in pairs
                    const float f = fminf(a.scale * a.cap_inv, FLT_MAX);       // never Inf, for a product may be 0
#pragma unroll
                    for (int n = 0; n < 128; n += 2) {
                        const float2 z = mul2(make_float2(x[n], x[n + 1]), twice(a.scale)), y = mul2(make_float2(x[n], x[n + 1]), twice(f)), t = mul2(y, y);
                        const float2 r = fma2(mul2(z, t), fma2(fma2(twice(-17.0f / 315.0f), t, twice(2.0f / 15.0f)), t, twice(-1.0f / 3.0f)), z);
                        x[n] = r.x, x[n + 1] = r.y;
                    }
                }
            }
            if (!whole) {
                // Bits of the keys that the row's token sees: of each cell, those up to its own place, and of these the window's and the first ones.
                const int bits = there.x | there.y << 2 | there.z << 4 | there.w << 6;
                uint32_t seen[kUnitCells];
#pragma unroll
                for (int j = 0; j < kUnitCells; ++j) {
                    const int from = block.cell_at((off + i) * kUnitCells + j) * kCell;
                    uint32_t m = low_bits(position + 1 - from);
                    if (a.window > 0) m &= ~low_bits(position + 1 - a.window - from) | low_bits(a.sinks - from);
                    seen[j] = bits >> j & 1 ? m : 0u;
                }
#pragma unroll
                for (int n = 0; n < 128; ++n) x[n] = seen[cell_of(n)] & 1u << token_of(n) ? x[n] : -INFINITY;
            }
            float mosts[4];                                     // in chains side by side
#pragma unroll
            for (int j = 0; j < 4; ++j) mosts[j] = fmaxf(x[j], x[4 + j]);
#pragma unroll
            for (int n = 8; n < 128; n += 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j) mosts[j] = max3(mosts[j], x[n + j], x[n + 4 + j]);
            }
            float most = fmaxf(max3(mosts[0], mosts[1], mosts[2]), mosts[3]);
            const float factor = kCap ? 1.0f : a.scale;
            most *= factor;
            // weights as in kv8.cu: 2^(score - top), top the largest score so far less kHeadroom, or up to kSlack less
            if (__any_sync(0xFFFFFFFFu, most > top + (kHeadroom + kSlack))) {
                const float next = fmaxf(top, most - kHeadroom), f = exp2_of(top - next);
                top = next;
                weight *= f;
                if (i > 0) {
#pragma unroll 1
                    for (int d = 0; d < kDim; d += 32) {
                        float o[32];
                        tmem_load(at_sums + d, o);
                        tmem_loaded();
#pragma unroll
                        for (int n = 0; n < 32; ++n) o[n] *= f;
                        tmem_store(at_sums + d, reinterpret_cast<const uint32_t*>(o));
                    }
                    tmem_stored();
                }
            }
            const float2 factors = make_float2(factor, factor), tops = make_float2(-top, -top);
            float2 sums[4] = {};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t out[32];
#pragma unroll
                for (int n = 0; n < 32; ++n) {
                    float2 z = fma2(make_float2(x[64 * half + 2 * n], x[64 * half + 2 * n + 1]), factors, tops);
                    z.x = exp2_of(z.x), z.y = exp2_of(z.y);
                    sums[n & 3] = add2(sums[n & 3], z);
                    const __half2 h = __floats2half2_rn(z.x, z.y);
                    out[n] = *reinterpret_cast<const uint32_t*>(&h);
                }
                tmem_store(at_scores + 32 * half, out);
                tmem_stored();
                fence_before();
                __syncwarp();
                if (lane == 0) arrive(&bars->p_full[tile][half]);
            }
            const float2 sum = add2(add2(sums[0], sums[1]), add2(sums[2], sums[3]));
            weight += sum.x + sum.y;
        }
        // ---- the piece's sums
        ok = ok && __all_sync(0xFFFFFFFFu, wait_parity(&bars->o_full[tile], pieces & 1u));
        ++pieces;
        fence_after();
        if (!ok) weight = __int_as_float(0x7FC00000);           // NaN
        const int64_t column = static_cast<int64_t>(s->h * a.group + row - token * a.group) * kDim;
        const bool mine = t < rows;
        if (!s->whole && mine) a.stats[static_cast<int64_t>(s->slot) * F::kRows + tile * kTileRows + t] = make_float2(top, weight);
        const float inverse = weight > 0.0f || weight != weight ? 1.0f / weight : 0.0f;
#pragma unroll 1
        for (int d0 = 0; d0 < kDim; d0 += 64) {
            float o[64];
            __syncwarp();
            tmem_load(at_sums + d0, o);
            tmem_load(at_sums + d0 + 32, o + 32);
            tmem_loaded();
            if (!mine) continue;
            if (!ok) {
#pragma unroll
                for (int n = 0; n < 64; ++n) o[n] = weight;
            }
            if (!s->whole) {
                float4* to = reinterpret_cast<float4*>(a.sums + (static_cast<int64_t>(s->slot) * F::kRows + tile * kTileRows + t) * kDim + d0);
#pragma unroll
                for (int n = 0; n < 16; ++n) to[n] = make_float4(o[4 * n], o[4 * n + 1], o[4 * n + 2], o[4 * n + 3]);
                continue;
            }
            uint32_t words[32], keep[2] = {0, 0};
#pragma unroll
            for (int n = 0; n < 32; ++n) {
                const __half2 h = __floats2half2_rn(o[2 * n] * inverse, o[2 * n + 1] * inverse);
                words[n] = *reinterpret_cast<const uint32_t*>(&h);
            }
            __half* to = a.y + (block.n0 + token) * a.ldy + column + d0;
            if (p.wide16) {
#pragma unroll
                for (int n = 0; n < 8; ++n) reinterpret_cast<uint4*>(to)[n] = make_uint4(words[4 * n], words[4 * n + 1], words[4 * n + 2], words[4 * n + 3]);
            } else {
                unsigned short* h = reinterpret_cast<unsigned short*>(to);
#pragma unroll
                for (int n = 0; n < 32; ++n) h[2 * n] = static_cast<unsigned short>(words[n]), h[2 * n + 1] = static_cast<unsigned short>(words[n] >> 16);
            }
            if (a.mask != nullptr) {
#pragma unroll
                for (int n = 0; n < 32; ++n) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&words[n]));
                    keep[n / 16] |= (fabsf(f.x) <= a.thr ? 0u : 1u) << (2 * n & 31) | (fabsf(f.y) <= a.thr ? 0u : 2u) << (2 * n & 31);
                }
                uint32_t* to_mask = a.mask + (block.n0 + token) * a.mask_stride + (column + d0) / 32;
                to_mask[0] = keep[0], to_mask[1] = keep[1];
            }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(&bars->piece_free[number % kPieces]);
    }
}

template <int kDim, bool kCap>
__global__ void __launch_bounds__(kThreads, 1) kv8_prompt_kernel(const __grid_constant__ PromptParams p) {
    using F = Form<kDim>;
    extern __shared__ unsigned char raw[];
    unsigned char* operands = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    Barriers* bars = reinterpret_cast<Barriers*>(operands + F::kOperands);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            barrier_init(&bars->q_full[i], F::kTiles == 2 ? 1 : 2);
            barrier_init(&bars->q_free[i], 1);
            barrier_init(&bars->s_full[i], 1);
            barrier_init(&bars->p_full[i][0], 4);
            barrier_init(&bars->p_full[i][1], 4);
            barrier_init(&bars->o_full[i], 1);
            barrier_init(&bars->k_full[i], 4);
            barrier_init(&bars->k_free[i], 1);
            barrier_init(&bars->v_full[i], 4);
            barrier_init(&bars->v_free[i], 1);
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            barrier_init(&bars->piece_full[i], 1);
            barrier_init(&bars->piece_free[i], 4 * F::kTiles + 4 + 1 + 2);      // softmax, codes, products, rows of q
        }
        barrier_init(&bars->drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    dev::programmatic_start();
    const uint32_t tmem = bars->tmem, queries = smem_u32(operands), keys = queries + F::kTiles * F::kQueryBytes, values = keys + F::kStages * F::kKeyBytes;
    if (threadIdx.x == 0) p.a.open[blockIdx.x] = make_int4(-1, 0, 0, 0);
    __syncthreads();
    if (warp < 4 * F::kTiles) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F::kSoftmaxRegs));
        softmax_role<kDim, kCap>(p, bars, tmem, warp >> 2);
    } else if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kSecondRegs));
    } else if (warp < 12) {
        if constexpr (F::kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kDecodeRegs));
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F::kDecodeRegs));
        decode_role<kDim>(p, bars, keys, values);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kOtherRegs));
        if (warp == 12) {
            if (elect_one()) product_role<kDim>(p, bars, queries, keys, values, tmem);
            __syncwarp();
        } else if (warp == 13) {
            piece_role<F::kRows>(p, bars);
            const int columns = p.a.heads * p.a.group * kDim;
            for (int b = blockIdx.x; b < p.a.B; b += gridDim.x) {       // tokens of requests without keys
                const Request rq = request_of(p.a, b);
                if (rq.cells > 0) continue;
                for (int n = rq.n0; n < rq.n0 + rq.n; ++n) {
                    for (int i = threadIdx.x & 31; i < columns; i += 32) p.a.y[n * p.a.ldy + i] = __ushort_as_half(0);
                    if (p.a.mask != nullptr)
                        for (int i = threadIdx.x & 31; i < columns / 32; i += 32) p.a.mask[n * p.a.mask_stride + i] = 0.0f <= p.a.thr ? 0u : 0xFFFFFFFFu;
                }
            }
        } else query_role<kDim>(p, bars, queries, warp - 14);
    }
    fence_before();
    __syncthreads();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// Joins the partial sums of a block that several CTAs have, in the order of its keys: a row to a warp.
constexpr int kJoinWarps = 8;

template <int kDim>
__global__ void __launch_bounds__(32 * kJoinWarps) kv8_prompt_join_kernel(const __grid_constant__ PromptParams p) {
    constexpr int kRows = Form<kDim>::kRows, kLanes = kDim / 4, kFours = kDim > 128 ? kDim / 128 : 1;
    dev::programmatic_start();
    const AttnParams& a = p.a;
    const int4 open = a.open[blockIdx.x];
    if (open.x < 0) return;
    const Block& block = p.blocks[open.x];
    const int row = blockIdx.y * kJoinWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31, mine = block.row0 + row;
    if (row >= block.rows) return;
    const int count = open.w - open.z / 2 + 1;
    float m = kLowest, wt = 0.0f;
    float4 sum[kFours] = {};
#pragma unroll 2
    for (int i = 0; i < count; ++i) {
        const int64_t from = (i == 0 ? open.z : 2 * (open.z / 2 + static_cast<int64_t>(i))) * kRows + row;
        const float2 st = a.stats[from];
        const float top = fmaxf(m, st.x), f = exp2_of(m - top), fs = exp2_of(st.x - top);
#pragma unroll
        for (int j = 0; j < kFours; ++j) {
            if (lane >= kLanes) continue;
            const float4 v = *reinterpret_cast<const float4*>(a.sums + from * kDim + 128 * j + 4 * lane);
            sum[j].x = sum[j].x * f + v.x * fs, sum[j].y = sum[j].y * f + v.y * fs, sum[j].z = sum[j].z * f + v.z * fs, sum[j].w = sum[j].w * f + v.w * fs;
        }
        wt = wt * f + st.y * fs;
        m = top;
    }
#pragma unroll
    for (int j = 0; j < kFours; ++j)
        if (lane < kLanes) store_result(a, block.n0 + mine / a.group, static_cast<int64_t>(open.y * a.group + mine % a.group) * kDim + 128 * j + 4 * lane, sum[j], wt);
}

template <int kDim, bool kCap>
spdp_status launch_form(PromptParams p, int device, int sms, cudaStream_t s) {
    using F = Form<kDim>;
    constexpr size_t kShared = 1024 + F::kOperands + sizeof(Barriers);
    static_assert(kShared <= 227 * 1024, "shared memory of a CTA");
    static std::mutex mu;
    static bool configured[64] = {};
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[device]) {
            SPDP_CUDA_TRY(cudaFuncSetAttribute(kv8_prompt_kernel<kDim, kCap>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kShared)));
            configured[device] = true;
        }
    }
    const int64_t rows = static_cast<int64_t>(p.a.N) * p.a.group;
    p.most_list = static_cast<int>(rows / F::kRows + p.a.B);
    const size_t sums = 2ull * sms * F::kRows * kDim * sizeof(float), stats = 2ull * sms * F::kRows * sizeof(float2), open = sms * sizeof(int4);
    void* scratch = nullptr;
    const spdp_status st = scratch_alloc(device, sums + stats + open + p.most_list * sizeof(Block) + 2 * sizeof(int), s, &scratch);
    if (st != SPDP_OK) return st;
    char* at = static_cast<char*>(scratch);
    p.a.sums = reinterpret_cast<float*>(at), p.a.stats = reinterpret_cast<float2*>(at + sums), p.a.open = reinterpret_cast<int4*>(at + sums + stats);
    p.blocks = reinterpret_cast<Block*>(at + sums + stats + open), p.totals = reinterpret_cast<int*>(p.blocks + p.most_list);
    cudaError_t e = cudaSuccess;
    if (p.a.B <= kShortRequests && p.most_list <= kShortList) p.totals = nullptr;
    else e = launch_programmatic(kv8_blocks_kernel<F::kRows>, dim3(1), kListThreads, 0, s, p);
    if (e == cudaSuccess) e = launch_programmatic(kv8_prompt_kernel<kDim, kCap>, dim3(static_cast<unsigned>(sms)), kThreads, kShared, s, p);
    if (e == cudaSuccess) e = launch_programmatic(kv8_prompt_join_kernel<kDim>, dim3(static_cast<unsigned>(sms), F::kRows / kJoinWarps), 32 * kJoinWarps, 0, s, p);
    const cudaError_t freed = cudaFreeAsync(scratch, s);
    SPDP_CUDA_TRY(e);
    SPDP_CUDA_TRY(freed);
    return SPDP_OK;
}

}  // namespace

spdp_status launch_kv8_prompt(const AttnParams& a, int head_dim, int device, int sms, cudaStream_t s) {
    PromptParams p = {};
    p.a = a;
    p.negative = a.scale < 0.0f;
    p.a.scale = fmaxf(fabsf(a.scale), 1.0e-30f);                // never 0: a masked score is -Inf, and stays it
    p.wide16 = rows_aligned16(a.y, a.ldy, 2);
    while ((1u << p.shift) < static_cast<unsigned>(a.group)) ++p.shift;
    p.magic = static_cast<uint32_t>((((1ull << p.shift) - a.group) << 32) / a.group + 1);
    switch (head_dim) {
        case 64: return a.cap > 0.0f ? launch_form<64, true>(p, device, sms, s) : launch_form<64, false>(p, device, sms, s);
        case 128: return a.cap > 0.0f ? launch_form<128, true>(p, device, sms, s) : launch_form<128, false>(p, device, sms, s);
        default: return a.cap > 0.0f ? launch_form<256, true>(p, device, sms, s) : launch_form<256, false>(p, device, sms, s);
    }
}

}  // namespace spdp
