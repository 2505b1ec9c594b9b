// Products on v_mfma_f32_32x32x16_bf16 (2.2 to 2.4 PFLOP/s on this device where 16x16x32 reaches 2.0 to 2.1) with their
// operands read from LDS ahead of them, and the stores of their sums (ffn_res.hip, ffn.hip).
#pragma once

#include "ffn_bf16.h"

namespace gsc {

typedef float floatx16 __attribute__((ext_vector_type(16)));

// 16 bytes a lane of a block of 1 KiB
__device__ __forceinline__ fbf16x8 res_frag(const uint8_t* blk) {
    return *reinterpret_cast<const fbf16x8*>(blk + (threadIdx.x & 63) * 16);
}
__device__ __forceinline__ floatx16 res_mma(fbf16x8 w, fbf16x8 x, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x, c, 0, 0, 0);
}

// f(constant 0), f(constant 1), ...
template <int N, typename F>
__device__ __forceinline__ void res_each(F f) {
    if constexpr (N > 0) {
        res_each<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// N products in groups of G: use(j, fragments of product j), the fragments read(j) from LDS a group ahead; after each
// group's products side(i), vector instructions of the group's share, VPM of them between two products.
template <int N, int G, int VPM, typename R, typename F, typename E>
__device__ __forceinline__ void res_stream(R read, F use, E side) {
    static_assert(N % G == 0, "whole groups");
    typedef decltype(read(0)) Reg;
    Reg f[2][G];
#pragma unroll
    for (int j = 0; j < G; ++j) f[0][j] = read(j);
    res_each<N / G>([&](auto I) {
        constexpr int i = decltype(I)::value;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (i + 1 < N / G) {
#pragma unroll
            for (int j = 0; j < G; ++j) f[(i + 1) & 1][j] = read((i + 1) * G + j);
        }
#pragma unroll
        for (int j = 0; j < G; ++j) use(i * G + j, f[i & 1][j]);
        side(I);
        // the order: the next group's reads, then a product and its share of vector instructions in turn
        __builtin_amdgcn_sched_group_barrier(0x100, i + 1 < N / G ? G * (int)(sizeof(Reg) / 16) : 0, 0);
#pragma unroll
        for (int j = 0; j < G; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (VPM) __builtin_amdgcn_sched_group_barrier(0x002, VPM, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    });
}

// A 32 x 32 tile of values as bfloat16 pairs (v[k]: registers 2 k, 2 k + 1 of a lane), to rows row0 .. below n and columns
// col0 .. below limit.  Lanes exchange halves (permlane32_swap: 16 bytes of one row each; permlane16_swap: four lanes a
// row), so that a store covers 16 rows by 64 bytes.  WHOLE: the tile lies inside; two store instructions.
template <bool WHOLE>
__device__ __forceinline__ void res_store(uint16_t* __restrict__ out, int64_t ld, int64_t row0, int64_t n, int64_t col0,
                                          int64_t limit, const uint32_t (&v)[8]) {
    uint32_t c[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const auto s = __builtin_amdgcn_permlane32_swap(v[4 * t + e], v[4 * t + 2 + e], false, false);
            c[t][e] = s[0];
            c[t][2 + e] = s[1];
        }
    RowVec<uint16_t>::Raw w[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const auto s = __builtin_amdgcn_permlane16_swap(c[0][e], c[1][e], false, false);
        w[0][e] = s[0];
        w[1][e] = s[1];
    }
    const int i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
    const int64_t at = col0 + 16 * (q & 1) + 8 * (q >> 1);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int64_t row = row0 + 16 * r + i;
        if (WHOLE || (row < n && at + 8 <= limit)) {
            *reinterpret_cast<RowVec<uint16_t>::Raw*>(out + row * ld + at) = w[r];
        } else if (row < n) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < limit) out[row * ld + at + e] = (uint16_t)(w[r][e >> 1] >> (16 * (e & 1)));
        }
    }
}

}  // namespace gsc
