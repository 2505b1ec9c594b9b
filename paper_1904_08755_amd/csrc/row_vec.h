// Rows of features as 16-byte pieces, for the row-wise operators (norm.hip, rotary.hip).
#pragma once

#include "conv_common.h"

namespace gsc {

typedef __bf16 rv_bf16x2 __attribute__((ext_vector_type(2)));
typedef float rv_floatx2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(rv_floatx2{lo, hi}, rv_bf16x2));
}

// 16 bytes of a row that may start at any element: one load or store, without the promise of a
// 16-byte address to the compiler.
template <typename T>
struct RowVec;
template <>
struct RowVec<float> {
    static constexpr int V = 4;
    typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ float get(const Raw& r, int e) { return __uint_as_float(r[e]); }
    static __device__ __forceinline__ Raw put(const float (&v)[V]) {
        Raw r;
#pragma unroll
        for (int e = 0; e < V; ++e) r[e] = __float_as_uint(v[e]);
        return r;
    }
};
template <>
struct RowVec<uint16_t> {
    static constexpr int V = 8;
    typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ float get(const Raw& r, int e) {
        return __uint_as_float(e & 1 ? r[e >> 1] & 0xffff0000u : r[e >> 1] << 16);
    }
    static __device__ __forceinline__ Raw put(const float (&v)[V]) {
        Raw r;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) r[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        return r;
    }
};

// Buffer loads (a bounds check instead of a branch): word 3 of the descriptor for 32-bit data, and an offset past any
// operand's end, which reads zeros.
constexpr int kBufFlags = 0x00020000;
constexpr uint32_t kBufNone = 0x80000000u;

// Elements [0, left) of 16 bytes, zeros behind them.  TAIL = false: left is 0 or at least V.
template <typename T, bool TAIL>
__device__ __forceinline__ typename RowVec<T>::Raw load_vec(const T* p, int64_t left) {
    typedef RowVec<T> R;
    typename R::Raw r = {0, 0, 0, 0};
    if (left >= R::V) {
        r = *reinterpret_cast<const typename R::Raw*>(p);
    } else if (TAIL && left > 0) {
        if constexpr (sizeof(T) == 4) {
            for (int e = 0; e < R::V; ++e)
                if (e < left) r[e] = __float_as_uint(p[e]);
        } else {
#pragma unroll
            for (int e = 0; e < R::V; ++e)
                if (e < left) r[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        }
    }
    return r;
}

// Elements [col, col + V) of a row of c >= V, zeros behind its end.  A piece that the end cuts is the row's last 16 bytes,
// shifted by as much in every lane (loads of its elements one by one take as long as the rest of a row).
template <typename T>
__device__ __forceinline__ typename RowVec<T>::Raw load_last(const T* x, int64_t col, int c) {
    constexpr int V = RowVec<T>::V;
    typedef typename RowVec<T>::Raw Raw;
    Raw r = {0, 0, 0, 0};
    if (col < c) r = *reinterpret_cast<const Raw*>(x + (col + V <= c ? col : c - V));
    if (col + V > c) {
        const int sh = (V - c % V) * 8 * (int)sizeof(T);   // 16 .. 112 bits (where col < c)
        const uint64_t lo = (uint64_t)r[1] << 32 | r[0], hi = (uint64_t)r[3] << 32 | r[2];
        const uint64_t a = sh >= 64 ? hi >> (sh & 63) : lo >> sh | hi << (64 - sh), b = sh >= 64 ? 0 : hi >> sh;
        r = Raw{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    }
    return r;
}

template <typename T, bool TAIL>
__device__ __forceinline__ void store_vec(T* p, int64_t left, const float (&v)[RowVec<T>::V]) {
    typedef RowVec<T> R;
    if (left >= R::V) {
        *reinterpret_cast<typename R::Raw*>(p) = R::put(v);
    } else if (TAIL) {
#pragma unroll
        for (int e = 0; e < R::V; ++e)
            if (e < left) store_out(&p[e], v[e]);
    }
}

// A matrix as row-major rows of ld elements, or in blocks of 128 rows by 32 columns, each one piece of memory (row-major
// inside), the blocks of 128 rows after each other: a step of 32 columns of a tile's rows is then contiguous, where a
// row-major one takes a piece of every row, a power of two apart for the usual widths, and most memory channels idle.
// Element (r, c) at p[(r / 128) ts + (r % 128) ld + (c / 32) gs + c % 32].
template <typename T>
struct RowMat {
    T* p;
    int64_t ld, gs, ts;
    // from row r (a multiple of the rows a tile takes) and column c (a multiple of 32) on
    __host__ __device__ __forceinline__ RowMat at(int64_t r, int64_t c) const {
        return {p + (r >> 7) * ts + (r & 127) * ld + (c >> 5) * gs, ld, gs, ts};
    }
};
template <typename T>
__host__ __device__ __forceinline__ RowMat<T> row_major(T* p, int64_t ld) {
    return {p, ld, 32, 128 * ld};
}
// columns: of all matrices that share the blocks of 128 rows
template <typename T>
__host__ __device__ __forceinline__ RowMat<T> row_blocks(T* p, int64_t columns) {
    return {p, 32, 4096, columns * 128};
}

}  // namespace gsc
