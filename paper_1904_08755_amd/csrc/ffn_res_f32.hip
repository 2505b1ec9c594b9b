// Feed-forward kernels for many rows of at most 128 channels in float32: a wave keeps 32 rows of X (and dY) in its registers
// and walks over the hidden columns, 32 at a time, while the weights pass through LDS.
//
// Everything between the weights and the outputs stays in registers.  v_mfma_f32_32x32x2_f32 takes the weights first, so lane
// (i, q) gets row i and the hidden columns 8 j + 4 q + e of a 32 x 32 tile in register 4 j + e; the sum of the next product
// may take its elements in any order, so these registers are that product's other operand as they are, if the
// weights' lanes read the same columns.  Against the tiles of ffn_f32.h: forward no hidden row is written, backward dX needs no
// second pass over dG and dU, and a row is read once instead of once per 64 hidden columns.
//
// Bound: the matrix cores (float32 at a sixteenth of the bfloat16 rate; the 32 x 32 x 2 instruction reaches 156 TFLOP/s on this
// device, the 16 x 16 x 4 one of the tiles 136).  120,011 rows, 64 channels, 256 hidden: forward 125 us (tiles 160), backward
// without the weights' gradients 235 us (tiles 300); without its stores 197, without the activation the same.  3,751 wave
// tiles over 1,024 SIMDs are four rounds of which 3.66 are full.
#include "ffn_res.h"

#include "ffn_act.h"
#include "ffn_f32.h"
#include "ffn_mma.h"

namespace gsc {

constexpr int kR32Threads = 256;
constexpr int kR32Rows = 128;

// A chunk of 32 hidden columns in LDS: K rows of 32 columns of Wg and of Wu, and 32 rows of K columns of Wd (K channels; zeros
// behind the matrices' ends).  The 16-byte pieces of a row are permuted by the row modulo 8, so that 32 lanes
// that read a piece of a row each meet distinct banks eight at a time.
template <int K, bool WHOLE>
struct R32Chunk {
    static constexpr int kUp = K * 128, kDown = 2 * K * 128, kBytes = 3 * K * 128;   // where Wu and Wd start
    static constexpr int N = K / 32;                                                // pieces a thread and matrix
    typedef RowVec<float>::Raw Raw;
    Raw g[N], u[N], d[N];

    // The chunk at hidden column c0.  Thread (r, c) of 32 x 8: piece c of row r (+ 32 s) of Wg and Wu, piece c (+ 8 s) of row r
    // of Wd; offsets in bytes are below 2^32 (at most 128 x 2^20 floats).
    __device__ __forceinline__ void fetch(const float* Wg, const float* Wu, const float* Wd, int ci, int f, int co, int c0) {
        const uint32_t r = threadIdx.x >> 3, c = threadIdx.x & 7;
        const uint32_t up = (r * (uint32_t)f + c * 4) * 4, down = (r * (uint32_t)co + c * 4) * 4;
#pragma unroll
        for (int s = 0; s < N; ++s) {
            const int64_t at = (int64_t)(32 * s) * f + c0;
            const int left = (int)r + 32 * s < ci ? f - c0 - (int)c * 4 : 0;
            g[s] = get_f32<WHOLE>(Wg + at, up, left);
            u[s] = get_f32<WHOLE>(Wu + at, up, left);
            d[s] = get_f32<WHOLE>(Wd + (int64_t)c0 * co + 32 * s, down, c0 + (int)r < f ? co - 32 * s - (int)c * 4 : 0);
        }
    }
    __device__ __forceinline__ void put(uint8_t* lds) const {
        const int r = threadIdx.x >> 3, c = ((threadIdx.x & 7) ^ (r & 7)) * 16;
#pragma unroll
        for (int s = 0; s < N; ++s) {
            uint8_t* up = lds + r * 128 + c + s * 4096;
            *reinterpret_cast<uint4*>(up) = uint4{g[s][0], g[s][1], g[s][2], g[s][3]};
            *reinterpret_cast<uint4*>(up + kUp) = uint4{u[s][0], u[s][1], u[s][2], u[s][3]};
            *reinterpret_cast<uint4*>(lds + kDown + r * (4 * K) + c + s * 128) = uint4{d[s][0], d[s][1], d[s][2], d[s][3]};
        }
    }
};

// One product's weights of a lane (i, q) from a matrix of rows of RB bytes at m.
// Across the rows: element (8 j + 4 q + e, i) of columns 32 t ..
template <int RB>
__device__ __forceinline__ float r32_col(const uint8_t* m, int i, int q, int j, int e, int t) {
    return *reinterpret_cast<const float*>(m + (4 * q + e) * RB + ((i >> 2) ^ (4 * q + e)) * 16 + (i & 3) * 4 + j * 8 * RB +
                                           t * 128);
}
// Along them: elements (i, 8 j + 4 q ..) of rows 32 t ..
template <int RB>
__device__ __forceinline__ floatx4 r32_row(const uint8_t* m, int i, int q, int j, int t) {
    return *reinterpret_cast<const floatx4*>(m + i * RB + ((2 * (j & 3) + q) ^ (i & 7)) * 16 + (j >> 2) * 128 + t * 32 * RB);
}

// A lane's part (row i) of 32 rows of c columns at m, `rows` of them valid, as the products take them
template <int K, bool WHOLE>
__device__ __forceinline__ void r32_load(const float* m, int64_t rows, int c, int i, int q, floatx4 (&x)[K / 8]) {
#pragma unroll
    for (int j = 0; j < K / 8; ++j) {
        const RowVec<float>::Raw r = get_f32<WHOLE>(m + 8 * j, (uint32_t)(i * c + 4 * q) * 4, i < rows ? c - 8 * j - 4 * q : 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = __uint_as_float(r[e]);
    }
}

// Waits for the rows' loads, which the compiler would move to the loop: there it would wait for them, and with them for every
// store before, each time.
template <int K>
__device__ __forceinline__ void r32_here(floatx4 (&x)[K / 8]) {
#pragma unroll
    for (int j = 0; j < K / 8; ++j) asm volatile("" : "+v"(x[j]));
}

// A 32 x 32 tile to `rows` rows of `cols` columns at out (ALL: to all of them).  Lanes i and i + 16 exchange pieces
// (permlane16_swap), so that a store covers 16 rows by 64 bytes.
template <bool ALL>
__device__ __forceinline__ void r32_store(float* out, int64_t ld, int64_t rows, int64_t cols, const floatx16& v) {
    typedef RowVec<float>::Raw Raw;
    const int i = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        Raw w[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[8 * t + e]), __float_as_uint(v[8 * t + 4 + e]),
                                                            false, false);
            w[0][e] = s[0];
            w[1][e] = s[1];
        }
        const int col = 16 * t + 8 * (g & 1) + 4 * (g >> 1);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = 16 * r + i;
            float* p = out + row * ld + col;
            if (ALL || (row < rows && col + 4 <= cols)) {
                *reinterpret_cast<Raw*>(p) = w[r];
            } else if (row < rows) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < cols) p[e] = __uint_as_float(w[r][e]);
            }
        }
    }
}

// A barrier for LDS alone: the hidden rows' stores and the next chunk's loads stay in flight.
__device__ __forceinline__ void r32_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    fb_barrier();
}

__device__ __forceinline__ floatx16 r32_mma(float w, float x, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(w, x, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 r32_zero() {
    floatx16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}

// G and U of a chunk
template <int K>
__device__ __forceinline__ void r32_up(const uint8_t* lds, int i, int q, const floatx4 (&x)[K / 8], floatx16& g, floatx16& u) {
    g = r32_zero();
    u = r32_zero();
#pragma unroll
    for (int j = 0; j < K / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            g = r32_mma(r32_col<128>(lds, i, q, j, e, 0), x[j][e], g);
            u = r32_mma(r32_col<128>(lds + K * 128, i, q, j, e, 0), x[j][e], u);
        }
}

template <int K, bool WHOLE, int ACT>
__global__ void __launch_bounds__(kR32Threads, 2)
k_ffn_fwd_rows(const float* __restrict__ X, int64_t n, int ci, const float* __restrict__ Wg, const float* __restrict__ Wu, int f,
               const float* __restrict__ Wd, int co, float* __restrict__ Y) {
    typedef R32Chunk<K, WHOLE> C;
    __shared__ __attribute__((aligned(16))) uint8_t lds[C::kBytes];
    const int i = threadIdx.x & 31, q = (threadIdx.x & 63) >> 5;
    const int64_t row0 = (int64_t)blockIdx.x * kR32Rows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 32;
    floatx4 x[K / 8];
    r32_load<K, WHOLE>(X + row0 * ci, n - row0, ci, i, q, x);
    C next;
    next.fetch(Wg, Wu, Wd, ci, f, co, 0);
    r32_here<K>(x);
    floatx16 y[K / 32];
#pragma unroll
    for (int t = 0; t < K / 32; ++t) y[t] = r32_zero();
    next.put(lds);
    for (int c0 = 0; c0 < f; c0 += 32) {
        r32_barrier();   // the chunk is there
        floatx16 g, u;
        r32_up<K>(lds, i, q, x, g, u);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float a, d;
            ffn_act<ACT, false, false>(g[e], a, d);
            g[e] = a * u[e];
        }
        __builtin_amdgcn_sched_barrier(0);   // (the next chunk's registers live while u's do not)
        next.fetch(Wg, Wu, Wd, ci, f, co, c0 + 32);
#pragma unroll
        for (int t = 0; t < K / 32; ++t)
            if (32 * t < co)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    y[t] = r32_mma(r32_col<4 * K>(lds + C::kDown, i, q, e >> 2, e & 3, t), g[e], y[t]);
        r32_barrier();   // all have read it
        next.put(lds);
    }
#pragma unroll
    for (int t = 0; t < K / 32; ++t) r32_store<false>(Y + row0 * co + 32 * t, co, n - row0, co - 32 * t, y[t]);
}

// H, dG and dU (row_blocks, columns up to fp) and, where wanted, dX.
template <int K, bool WHOLE, int ACT>
__global__ void __launch_bounds__(kR32Threads, K <= 64 ? 2 : 1)
k_ffn_bwd_rows(const float* __restrict__ X, const float* __restrict__ dY, int64_t n, int ci, const float* __restrict__ Wg,
               const float* __restrict__ Wu, int f, const float* __restrict__ Wd, int co, int fp, RowMat<float> H,
               RowMat<float> dG, RowMat<float> dU, float* __restrict__ dX) {
    typedef R32Chunk<K, WHOLE> C;
    __shared__ __attribute__((aligned(16))) uint8_t lds[C::kBytes];
    const int i = threadIdx.x & 31, q = (threadIdx.x & 63) >> 5;
    const int64_t row0 = (int64_t)blockIdx.x * kR32Rows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 32, rows = n - row0;
    floatx4 x[K / 8], y[K / 8];
    r32_load<K, WHOLE>(X + row0 * ci, n - row0, ci, i, q, x);
    r32_load<K, WHOLE>(dY + row0 * co, n - row0, co, i, q, y);
    C next;
    next.fetch(Wg, Wu, Wd, ci, f, co, 0);
    r32_here<K>(x);
    r32_here<K>(y);
    floatx16 dx[K / 32];
#pragma unroll
    for (int t = 0; t < K / 32; ++t) dx[t] = r32_zero();
    next.put(lds);
    for (int c0 = 0; c0 < fp; c0 += 32) {
        r32_barrier();   // the chunk is there
        floatx16 g, u, d = r32_zero();
        r32_up<K>(lds, i, q, x, g, u);
#pragma unroll
        for (int j = 0; j < K / 8; ++j) {
            const floatx4 w = r32_row<4 * K>(lds + C::kDown, i, q, j, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) d = r32_mma(w[e], y[j][e], d);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float a, s;
            ffn_act<ACT, true, false>(g[e], a, s);
            g[e] = d[e] * u[e] * s;
            u[e] = a * u[e];
            d[e] = d[e] * a;
        }
        // before the stores, which the wait for it would include (neither is conditional, so that the compiler can count
        // them: behind the last chunk zeros are fetched, and rows behind the last one are stored to the blocks)
        __builtin_amdgcn_sched_barrier(0);
        next.fetch(Wg, Wu, Wd, ci, f, co, c0 + 32);
        __builtin_amdgcn_sched_barrier(0);
        r32_store<true>(H.at(row0, c0).p, 32, 0, 0, u);
        r32_store<true>(dG.at(row0, c0).p, 32, 0, 0, g);
        r32_store<true>(dU.at(row0, c0).p, 32, 0, 0, d);
        if (dX) {
#pragma unroll
            for (int t = 0; t < K / 32; ++t)
                if (32 * t < ci)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const floatx4 wg = r32_row<128>(lds, i, q, j, t), wu = r32_row<128>(lds + C::kUp, i, q, j, t);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            dx[t] = r32_mma(wg[e], g[4 * j + e], dx[t]);
                            dx[t] = r32_mma(wu[e], d[4 * j + e], dx[t]);
                        }
                    }
        }
        r32_barrier();   // all have read it
        next.put(lds);
    }
    if (dX) {
#pragma unroll
        for (int t = 0; t < K / 32; ++t) r32_store<false>(dX + row0 * ci + 32 * t, ci, rows, ci - 32 * t, dx[t]);
    }
}

// f(K, WHOLE, activation as constants).  (With the activation as a switch in the loop, k_ffn_bwd_rows<64> spills, and the wait
// for a reload is one for all stores before it.)
template <typename F>
static void r32_with(int ci, int f, int co, int act, F run) {
    const int c = ci > co ? ci : co;
    auto acts = [&](auto K, auto WHOLE) {
        switch (act) {
            case GSC_GATE_RELU: run(K, WHOLE, std::integral_constant<int, GSC_GATE_RELU>{}); break;
            case GSC_GATE_SIGMOID: run(K, WHOLE, std::integral_constant<int, GSC_GATE_SIGMOID>{}); break;
            case GSC_GATE_GELU: run(K, WHOLE, std::integral_constant<int, GSC_GATE_GELU>{}); break;
            case GSC_GATE_GELU_TANH: run(K, WHOLE, std::integral_constant<int, GSC_GATE_GELU_TANH>{}); break;
            default: run(K, WHOLE, std::integral_constant<int, GSC_GATE_SILU>{}); break;
        }
    };
    auto with = [&](auto K) {
        if (ci % 4 == 0 && f % 4 == 0 && co % 4 == 0) acts(K, std::true_type{});
        else acts(K, std::false_type{});
    };
    if (c <= 32) with(std::integral_constant<int, 32>{});
    else if (c <= 64) with(std::integral_constant<int, 64>{});
    else if (c <= 96) with(std::integral_constant<int, 96>{});
    else with(std::integral_constant<int, 128>{});
}

void res_fwd(const float* X, int64_t n, int ci, const float* Wg, const float* Wu, int f, const float* Wd, int co, int act,
             float* Y, hipStream_t s) {
    r32_with(ci, f, co, act, [&](auto K, auto WHOLE, auto ACT) {
        auto* kern = k_ffn_fwd_rows<decltype(K)::value, decltype(WHOLE)::value, decltype(ACT)::value>;
        hipLaunchKernelGGL(kern, dim3((unsigned)((n + kR32Rows - 1) / kR32Rows)), dim3(kR32Threads), 0, s, X, n, ci, Wg, Wu, f,
                           Wd, co, Y);
    });
}

void res_bwd(const float* X, const float* dY, int64_t n, int ci, const float* Wg, const float* Wu, int f, const float* Wd,
             int co, int act, int fp, RowMat<float> H, RowMat<float> dG, RowMat<float> dU, float* dX, hipStream_t s) {
    r32_with(ci, f, co, act, [&](auto K, auto WHOLE, auto ACT) {
        auto* kern = k_ffn_bwd_rows<decltype(K)::value, decltype(WHOLE)::value, decltype(ACT)::value>;
        hipLaunchKernelGGL(kern, dim3((unsigned)((n + kR32Rows - 1) / kR32Rows)), dim3(kR32Threads), 0, s, X, dY, n, ci, Wg,
                           Wu, f, Wd, co, fp, H, dG, dU, dX);
    });
}

}  // namespace gsc
