// Device helpers shared by the operators around the projections (lora.cu, heads.cu, kv4.cu): fp16 matrix products on
// register fragments and the waits of programmatic launches.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace spdp {
namespace dev {

// The next kernel of the stream may be set up now; what earlier kernels wrote or still read is touched after the wait.
__device__ __forceinline__ void programmatic_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// d[16][8] += a[16][16] b[16][8], fp16 in, fp32 sums.  Lane (g, c) = (lane / 4, lane % 4) holds a's rows g and g + 8 (a0/a2 and
// a1/a3), b's column g, and d's rows g (d0, d1) and g + 8 (d2, d3), columns 2 c and 2 c + 1.  Which k a register's pair stands for
// is the caller's choice, as long as a and b agree: the loads below give a lane whole 16-byte runs of a row.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with sums that start from `from`.
__device__ __forceinline__ void mma_f16_from(float (&d)[4], float from0, float from1, float from2, float from3, uint32_t a0, uint32_t a1, uint32_t a2,
                                             uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(from0), "f"(from1), "f"(from2), "f"(from3));
}

// Elements k .. k + 7 of a row (k a multiple of 8) of which those from `limit` on are zeros, without a branch, so that many such
// loads are on their way at once.  kAlign: 16, 4 or 2 bytes, what every row's address is a multiple of; with 16 the elements up
// to the next multiple of 8 are read too and come back as they are.
template <int kAlign>
__device__ __forceinline__ uint4 load8(const __half* row, int k, int limit) {
    if constexpr (kAlign == 16) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (k < limit) v = *reinterpret_cast<const uint4*>(row + k);
        return v;
    } else if constexpr (kAlign == 4) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = k + 2 * i;
            uint32_t both = 0, one = 0;
            if (at + 1 < limit) both = *reinterpret_cast<const uint32_t*>(row + at);
            if (at + 1 == limit) one = __half_as_ushort(row[at]);
            w[i] = both | one;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        // Three whole words lie inside the eight elements, one or two elements from the first; besides them the first element, and
        // the second or the last.
        const int odd = static_cast<int>(reinterpret_cast<uintptr_t>(row + k) >> 1 & 1), side = odd ? k + 7 : k + 1;
        uint32_t first = 0, other = 0, w[3];
        if (k < limit) first = __half_as_ushort(row[k]);
        if (side < limit) other = __half_as_ushort(row[side]);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int at = k + 2 - odd + 2 * i;
            uint32_t both = 0, one = 0;
            if (at + 1 < limit) both = *reinterpret_cast<const uint32_t*>(row + at);
            if (at + 1 == limit) one = __half_as_ushort(row[at]);
            w[i] = both | one;
        }
        const uint32_t take = odd ? 0x5432 : 0x3210;            // halves (second of a, first of b); or a
        uint4 v;
        v.x = __byte_perm(first, odd ? w[0] : other, 0x5410);
        v.y = __byte_perm(w[0], w[1], take);
        v.z = __byte_perm(w[1], w[2], take);
        v.w = __byte_perm(w[2], other, take);
        return v;
    }
}
// Zeros in the elements from `limit` on of what stands for elements k .. k + 7.
__device__ __forceinline__ void cut8(uint4& v, int k, int limit) {
    auto keep = [&](int i) { return k + 2 * i + 1 < limit ? 0xFFFFFFFFu : k + 2 * i < limit ? 0x0000FFFFu : 0u; };
    v.x &= keep(0), v.y &= keep(1), v.z &= keep(2), v.w &= keep(3);
}

// Eight consecutive values of a row as fp32, in 16-byte loads where the address allows them.
template <typename T, bool kWide>
__device__ __forceinline__ void load_floats(const T* at, float (&x)[8]) {
    if constexpr (kWide && sizeof(T) == 2) {
        const uint4 v = *reinterpret_cast<const uint4*>(at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    } else if constexpr (kWide) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 v = reinterpret_cast<const float4*>(at)[i];
            x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 2) x[i] = __half2float(at[i]);
            else x[i] = at[i];
        }
    }
}

// Eight values, rounded to fp16, into a row.
template <bool kWide>
__device__ __forceinline__ void store_halves(__half* at, const float (&x)[8]) {
    if constexpr (kWide) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = __float2half_rn(x[i]);
    }
}

}  // namespace dev

// What the addresses of rows `ld` elements of `size` bytes apart are multiples of, 16 at most.
inline int rows_alignment(const void* p, int64_t ld, int64_t size) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * size) | 16u;
    return static_cast<int>(bits & (~bits + 1));
}
inline bool rows_aligned16(const void* p, int64_t ld, int64_t size) { return rows_alignment(p, ld, size) == 16; }

// A launch that may be set up while the kernel before it still runs (programmatic_start() in the kernel waits for it).
template <typename... Formal, typename... Actual>
cudaError_t launch_programmatic(void (*kernel)(Formal...), dim3 grid, dim3 threads, size_t shared_bytes, cudaStream_t s, const Actual&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = shared_bytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
}  // namespace spdp
