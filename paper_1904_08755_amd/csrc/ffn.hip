// Gated feed-forward block of feature rows, forward and backward.
//
//   G = X Wg,  U = X Wu,  H = act(G) * U,  Y = H Wd
//   dH = dY Wd^T,  dG = dH U act'(G),  dU = dH act(G)
//   dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU,  dWd = H^T dY
//
// Products run on the matrix cores with float32 sums.  The backward pass works G and U out again from X (a third more products
// than reading them back, but the forward pass need not write them nor the program keep them: at 256 channels and 1,024
// hidden ones their two arrays would be eight times the bytes of X).  Which kernels take a call:
//   a few rows           k_ffn_few, twice;
//   many rows, narrow    rows stay in registers while the weights pass through LDS (ffn_res.hip, ffn_res_f32.hip);
//   else                 tiles: k_ffn_up (both projections with the activation; G and U never leave the registers) and
//                        k_ffn_gemm; backward k_ffn_mid (G, U and dH of a tile; stores H, dG and dU) and k_ffn_gemm for dX.
// The weights' gradients are k_ffn_dw over row chunks and k_ffn_dw_sum, which adds the chunks in order: every result is
// bit-reproducible.
//
// bfloat16: G, U, dH and all sums stay in float32; H (but for a few rows), dG and dU are rounded to bfloat16 once, as the
// matrix cores take them, and the results once as they are stored.  Its tiles copy operands straight into LDS (ffn_bf16.h),
// which takes rows of whole 16-byte pieces at 16-byte addresses: operands that are not are copied into the workspace first,
// their rows padded with zeros (k_ffn_pad; the weights and at most two passes over rows, against kernels that would load
// element by element).  float32 tiles (ffn_f32.h) take any address.
#include "ffn_act.h"
#include "ffn_bf16.h"
#include "ffn_f32.h"
#include "ffn_mma.h"
#include "ffn_res.h"

namespace gsc {

constexpr int kFfnMaxWidth = 1 << 20;
constexpr int kFfnFewRows = 4;                          // rows up to which k_ffn_few runs

// Four consecutive columns of a row from each of two neighbouring 16-column blocks, as a lane holds them (columns col ..
// and col + 16 .., col = 32 c + 4 q), stored below `limit` to the row at p.  bfloat16: lanes q and q + 1 exchange
// halves (permlane16_swap) so that each has 16 bytes of one block: a store of 64 lanes covers 16 rows by
// 64 bytes.  (8 bytes a lane in 32-byte pieces: k_ffn_mid spent as long storing as on everything else.)
__device__ __forceinline__ void store_pair(float* p, int64_t col, int64_t limit, bool on, const float (&u)[4],
                                           const float (&v)[4]) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const float (&w)[4] = b ? v : u;
        const int64_t at = col + 16 * b;
        if (on && at + 4 <= limit) {
            *reinterpret_cast<floatx4u*>(p + at) = floatx4u{w[0], w[1], w[2], w[3]};
        } else if (on) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at + e < limit) p[at + e] = w[e];
        }
    }
}
__device__ __forceinline__ void store_pair(uint16_t* p, int64_t col, int64_t limit, bool on, const float (&u)[4],
                                           const float (&v)[4]) {
    const int q = (threadIdx.x & 63) >> 4;
    const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(u[0], u[1]), pack_bf16(v[0], v[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(u[2], u[3]), pack_bf16(v[2], v[3]), false, false);
    const RowVec<uint16_t>::Raw w = {lo[0], hi[0], lo[1], hi[1]};
    const int64_t at = col - 4 * q + 16 * (q & 1) + 8 * (q >> 1);
    if (on && at + 8 <= limit) {
        *reinterpret_cast<RowVec<uint16_t>::Raw*>(p + at) = w;
    } else if (on) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < limit) p[at + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}

// ---------------------------------------------------------------------------
// what happens to a tile's sums: lane (i, q) of a wave holds row 16 mi + i of its rows and columns 16 ni + 4 q ..
// of its columns
// ---------------------------------------------------------------------------
__device__ __forceinline__ int ffn_i() { return threadIdx.x & 15; }
__device__ __forceinline__ int ffn_q() { return (threadIdx.x & 63) >> 4; }

template <int MT, int NT>
__device__ __forceinline__ void zero_acc(floatx4 (&acc)[MT][NT]) {
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
}

// the sums themselves, to rows below n and columns below nn
template <typename T, int MT, int NT>
__device__ __forceinline__ void store_tile(const floatx4 (&acc)[MT][NT], int64_t row0, int64_t col0, int64_t n, int64_t nn,
                                           T* __restrict__ out, int64_t ld) {
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) {
        const int64_t row = row0 + 16 * mi + ffn_i();
#pragma unroll
        for (int ni = 0; ni < NT; ni += 2) {
            const float u[4] = {acc[mi][ni][0], acc[mi][ni][1], acc[mi][ni][2], acc[mi][ni][3]};
            const float v[4] = {acc[mi][ni + 1][0], acc[mi][ni + 1][1], acc[mi][ni + 1][2], acc[mi][ni + 1][3]};
            store_pair(out + row * ld, col0 + 16 * ni + 4 * ffn_q(), nn, row < n, u, v);
        }
    }
}

// H, dG and dU lie in blocks of 128 rows by 32 columns (row_blocks): a wave's 32 hidden columns are one block's.
// H from gates (blocks 0, 1) and their partners (blocks 2, 3)
template <typename T, int MT>
__device__ __forceinline__ void store_hidden(const floatx4 (&acc)[MT][4], int64_t row0, int64_t col0, int64_t n, int act,
                                             const RowMat<T>& H) {
    with_act(act, [&](auto ACT) {
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
            const int64_t row = row0 + 16 * mi + ffn_i();
            float h[2][4];
#pragma unroll
            for (int ni = 0; ni < 2; ++ni)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, d;
                    ffn_act<decltype(ACT)::value, false, sizeof(T) == 2>(acc[mi][ni][e], a, d);
                    h[ni][e] = a * acc[mi][ni + 2][e];
                }
            store_pair(H.at(row, col0).p, 4 * ffn_q(), 32, row < n, h[0], h[1]);
        }
    });
}

// H, dG and dU from gates, partners and dH
template <typename T, int MT>
__device__ __forceinline__ void store_mid(const floatx4 (&acc)[MT][4], const floatx4 (&dh)[MT][2], int64_t row0,
                                          int64_t col0, int64_t n, int act, const RowMat<T>& H, const RowMat<T>& dG,
                                          const RowMat<T>& dU) {
    with_act(act, [&](auto ACT) {
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
            const int64_t row = row0 + 16 * mi + ffn_i();
            float h[2][4], dg[2][4], du[2][4];
#pragma unroll
            for (int ni = 0; ni < 2; ++ni)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, d;
                    ffn_act<decltype(ACT)::value, true, sizeof(T) == 2>(acc[mi][ni][e], a, d);
                    const float up = acc[mi][ni + 2][e], g = dh[mi][ni][e];
                    h[ni][e] = a * up;
                    dg[ni][e] = g * up * d;
                    du[ni][e] = g * a;
                }
            store_pair(H.at(row, col0).p, 4 * ffn_q(), 32, row < n, h[0], h[1]);
            store_pair(dG.at(row, col0).p, 4 * ffn_q(), 32, row < n, dg[0], dg[1]);
            store_pair(dU.at(row, col0).p, 4 * ffn_q(), 32, row < n, du[0], du[1]);
        }
    });
}

// ---------------------------------------------------------------------------
// float32 kernels: tiles of 32 MT rows
// ---------------------------------------------------------------------------
// H (columns behind f zero) of a tile by 64 hidden columns.
template <int MT, bool WHOLE>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_up_f32(const float* __restrict__ X, int64_t n, int ci, const float* __restrict__ Wg, const float* __restrict__ Wu,
             int f, int act, RowMat<float> H, int nf) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, 4>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nf * (32 * MT);
    const int c0 = (int)(u % nf) * 64, wave = threadIdx.x >> 6;
    floatx4 acc[MT][4];
    zero_acc(acc);
    tile_product<true, false, MT, 4, true, WHOLE>({row_major(X + r0 * ci, ci), nullptr, n - r0, ci},
                                           {row_major(Wg + c0, f), Wu + c0, f - c0, ci}, lds, acc);
    store_hidden(acc, r0 + 16 * MT * (wave >> 1), c0 + 32 * (wave & 1), n, act, H);
}

// Out (n x co) = A1 B1 (+ A2 B2 where A2 is given) over k: A rows of the reduction (KC), B (row-major) either way.
template <bool BKC, int MT, int NT, bool WHOLE>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_gemm_f32(RowMat<const float> A1, RowMat<const float> A2, int64_t n, int64_t k, const float* __restrict__ B1,
               const float* __restrict__ B2, int64_t ldb, int co, float* __restrict__ Out, int nc) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, NT>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nc * (32 * MT);
    const int c0 = (int)(u % nc) * (32 * NT), wave = threadIdx.x >> 6;
    floatx4 acc[MT][NT];
    zero_acc(acc);
    for (int s = 0; s < 2; ++s) {
        const RowMat<const float> A = s ? A2 : A1;
        const float* B = s ? B2 : B1;
        if (!A.p) break;
        tile_product<true, BKC, MT, NT, false, WHOLE>({A.at(r0, 0), nullptr, n - r0, k},
                                               {row_major(BKC ? B + (int64_t)c0 * ldb : B + c0, ldb), nullptr, co - c0, k},
                                               lds, acc);
    }
    store_tile(acc, r0 + 16 * MT * (wave >> 1), c0 + 16 * NT * (wave & 1), n, co, Out, co);
}

// H, dG and dU of a tile by 64 hidden columns.
template <int MT, bool WHOLE>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_mid_f32(const float* __restrict__ X, const float* __restrict__ dY, int64_t n, int ci, int co,
              const float* __restrict__ Wg, const float* __restrict__ Wu, const float* __restrict__ Wd, int f, int act,
              RowMat<float> H, RowMat<float> dG, RowMat<float> dU, int nf) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, 4>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nf * (32 * MT);
    const int c0 = (int)(u % nf) * 64, wave = threadIdx.x >> 6;
    floatx4 acc[MT][4], dh[MT][2];
    zero_acc(acc);
    zero_acc(dh);
    tile_product<true, false, MT, 4, true, WHOLE>({row_major(X + r0 * ci, ci), nullptr, n - r0, ci},
                                           {row_major(Wg + c0, f), Wu + c0, f - c0, ci}, lds, acc);
    tile_product<true, true, MT, 2, false, WHOLE>({row_major(dY + r0 * co, co), nullptr, n - r0, co},
                                           {row_major(Wd + (int64_t)c0 * co, co), nullptr, f - c0, co}, lds, dh);
    store_mid(acc, dh, r0 + 16 * MT * (wave >> 1), c0 + 32 * (wave & 1), n, act, H, dG, dU);
}

// One product of k_ffn_dw: out (m x nn) = A^T B over the rows.
template <typename T>
struct DwSide {
    RowMat<const T> A, B;
    int m, nn;
    int tn, tiles;     // column tiles, all tiles (0: the product is not wanted)
    int64_t part;      // where its sums start in a chunk's partial sums
};

// Partial sums of a tile of 32 MT x 32 NT of one product over a chunk's rows
template <int MT, int NT, bool WHOLE>
__device__ __forceinline__ void dw_tile_f32(const DwSide<float>& p, int t, int64_t r0, int64_t rows, uint8_t* lds, float* out) {
    const int m0 = t / p.tn * (32 * MT), c0 = t % p.tn * (32 * NT), wave = threadIdx.x >> 6;
    floatx4 acc[MT][NT];
    zero_acc(acc);
    tile_product<false, false, MT, NT, false, WHOLE>({p.A.at(r0, m0), nullptr, p.m - m0, rows},
                                              {p.B.at(r0, c0), nullptr, p.nn - c0, rows}, lds, acc);
    store_tile(acc, m0 + 16 * MT * (wave >> 1), c0 + 16 * NT * (wave & 1), p.m, p.nn, out + p.part, p.nn);
}

// Partial sums of both products over the rows of a chunk, in tiles of 32 M0 channels by 128 hidden columns and of 128 hidden
// columns by 32 N1 channels.  120,011 rows, 64 channels, 256 hidden: 138 us (tiles of 64 x 64: 166), the matrix cores
// busy 59 % of it; more blocks change nothing, what counts is the 447 MB from beyond the L2s.
template <int M0, int N1, bool WHOLE>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_dw_f32(DwSide<float> p0, DwSide<float> p1, int64_t n, int64_t chunk, int64_t per_chunk, float* __restrict__ part) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<(M0 > N1 ? M0 : N1), 4>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int tiles = p0.tiles + p1.tiles;
    const int64_t s = u / tiles, r0 = s * chunk, rows = n - r0 < chunk ? n - r0 : chunk;
    const int t = (int)(u - s * tiles);
    if (t < p0.tiles) dw_tile_f32<M0, 4, WHOLE>(p0, t, r0, rows, lds, part + s * per_chunk);
    else dw_tile_f32<4, N1, WHOLE>(p1, t - p0.tiles, r0, rows, lds, part + s * per_chunk);
}

// ---------------------------------------------------------------------------
// bfloat16 kernels: operands with rows of whole 16-byte pieces (ld: their strides)
// ---------------------------------------------------------------------------
// Copies of up to five matrices with their rows padded to whole pieces.
struct FfnPad {
    const uint16_t* src[5];
    uint16_t* dst[5];
    int cols[5], ld[5];
    int64_t end[5];   // pieces of the matrices up to and with this one
    int count;
};
__global__ void __launch_bounds__(kFfnThreads) k_ffn_pad(FfnPad p) {
    const int64_t total = p.end[p.count - 1];
    for (int64_t i = (int64_t)blockIdx.x * kFfnThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kFfnThreads) {
        const uint16_t* src = p.src[0];
        uint16_t* dst = p.dst[0];
        int cols = p.cols[0], ld = p.ld[0];
        int64_t at = i;
#pragma unroll
        for (int m = 1; m < 5; ++m)
            if (m < p.count && i >= p.end[m - 1]) {
                src = p.src[m];
                dst = p.dst[m];
                cols = p.cols[m];
                ld = p.ld[m];
                at = i - p.end[m - 1];
            }
        const int64_t row = at / (ld / 8);
        const int c = (int)(at - row * (ld / 8)) * 8;
        const RowVec<uint16_t>::Raw v = cols < 8 ? load_vec<uint16_t, true>(src + row * cols + c, cols - c)
                                                 : load_last(src + row * cols, c, cols);
        *reinterpret_cast<uint4*>(dst + at * 8) = uint4{v[0], v[1], v[2], v[3]};
    }
}

// H of a tile of 32 MT rows by 64 hidden columns.
template <int MT>
__global__ void __launch_bounds__(256, 2)
k_ffn_up_bf16(const uint16_t* __restrict__ X, int64_t ldx, int64_t n, int ci, const uint16_t* __restrict__ Wg,
              const uint16_t* __restrict__ Wu, int64_t ldw, int f, int act, RowMat<uint16_t> H, int nf) {
    typedef FbShape<2, 2, MT, 4> S;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::LDS];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nf * S::BM;
    const int c0 = (int)(u % nf) * 64, wave = threadIdx.x >> 6;
    floatx4 acc[MT][4];
    zero_acc(acc);
    fb_product<2, 2, MT, 4, FB_KC, FB_MC, true>({row_major(X + r0 * ldx, ldx), n - r0}, {row_major(Wg + c0, ldw), f - c0},
                                                Wu + c0, ci, lds, acc);
    store_hidden(acc, r0 + 16 * MT * (wave >> 1), c0 + 32 * (wave & 1), n, act, H);
}

// Out (n x co, rows as they are) = A1 B1 (+ A2 B2 where A2 is given) over k.
template <int WM, int WN, int MT, FbLay BL>
__global__ void __launch_bounds__(256, 2)
k_ffn_gemm_bf16(RowMat<const uint16_t> A1, RowMat<const uint16_t> A2, int64_t n, int64_t k, const uint16_t* __restrict__ B1,
                const uint16_t* __restrict__ B2, int64_t ldb, int co, uint16_t* __restrict__ Out, int nc) {
    typedef FbShape<WM, WN, MT, 4> S;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::LDS];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nc * S::BM;
    const int c0 = (int)(u % nc) * S::BN, wave = threadIdx.x >> 6;
    floatx4 acc[MT][4];
    zero_acc(acc);
    for (int s = 0; s < 2; ++s) {
        const RowMat<const uint16_t> A = s ? A2 : A1;
        const uint16_t* B = s ? B2 : B1;
        if (!A.p) break;
        if (s) fb_barrier();   // the first product's last reads
        fb_product<WM, WN, MT, 4, FB_KC, BL>({A.at(r0, 0), n - r0},
                                             {row_major(BL == FB_KC ? B + (int64_t)c0 * ldb : B + c0, ldb), co - c0}, nullptr, k,
                                             lds, acc);
    }
    store_tile(acc, r0 + 16 * MT * (wave / WN), c0 + 64 * (wave % WN), n, co, Out, co);
}

// Out (n x co, at most 256) = A1 B1 + A2 B2 for KC operands in tiles of 256 x 256: eight waves of 64 x 128
// (v_mfma_f32_32x32x16_bf16), a ring of four stages of 32 reduction elements, each an array of its own: the operands are
// plain reads, which the compiler starts ahead of the products without waiting for copies into other stages.  Bound: about as
// much time in the copies as in the products (300,000 rows, 256 columns, 2 x 1,024 elements: 385 us; without the copies 288,
// without the products 368).
__global__ void __launch_bounds__(512, 1)
k_ffn_gemm_kc(RowMat<const uint16_t> A1, RowMat<const uint16_t> A2, int64_t n, int64_t k, const uint16_t* __restrict__ B1,
              const uint16_t* __restrict__ B2, int64_t ldb, int co, uint16_t* __restrict__ Out) {
    constexpr int TN = 4;   // 32-column tiles of a wave
    constexpr int BN = 64 * TN, STAGE = (256 + BN) * 64;
    typedef FbCopy<FB_KC, 256, 8, true> CA;
    typedef FbCopy<FB_KC, BN, 8, true> CB;
    constexpr int LD = CA::N + CB::N;
    __shared__ __attribute__((aligned(1024))) uint8_t slot0[STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t slot1[STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t slot2[STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t slot3[STAGE];
    auto slot = [&](auto N) -> uint8_t* {
        constexpr int s = decltype(N)::value % 4;
        return s == 0 ? slot0 : (s == 1 ? slot1 : (s == 2 ? slot2 : slot3));
    };
    const int64_t r0 = xcd_unit(blockIdx.x, gridDim.x) * 256;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const FbSide a1{A1.at(r0, 0), n - r0}, a2{A2.at(r0, 0), n - r0};
    const FbSide b1{row_major(B1, ldb), co}, b2{row_major(B2, ldb), co};
    CA ca;
    CB cb;
    ca.start(a1, wave);
    cb.start(b1, wave);
    const int half = (int)((k + 31) / 32), steps = 2 * half;
    auto issue = [&](int s, uint8_t* dst) {
        const bool second = s >= half;
        const int64_t k0 = (int64_t)(second ? s - half : s) * 32;
        ca.issue(second ? a2 : a1, k0, k, dst, wave);
        cb.issue(second ? b2 : b1, k0, k, dst + CA::BYTES, wave);
    };
    const int i = threadIdx.x & 31, h = (threadIdx.x & 63) >> 5;
    const int at = i * 64 + ((h ^ ((i >> 2) & 3)) * 16);   // elements 8 h .. of row i; 16 + 8 h .. at ^ 32
    floatx16 acc[2][TN];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) acc[a][b] = floatx16{};
    // During step s the copies of step s + 4 are started into the stage that step s's operands came from, the operands of
    // step s + 1 are read, and the products of step s run on those read during step s - 1.
    fbf16x8 fa[2][2][2], fb[2][2][TN];   // of even and odd steps: 16 reduction elements twice
    auto read = [&](auto N, fbf16x8 (&a)[2][2], fbf16x8 (&b)[2][TN]) {
        const uint8_t* la = slot(N) + wm * 4096;
        const uint8_t* lb = slot(N) + CA::BYTES + wn * TN * 2048;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
            for (int m = 0; m < 2; ++m) a[kk][m] = *reinterpret_cast<const fbf16x8*>(la + m * 2048 + (at ^ (32 * kk)));
#pragma unroll
            for (int t = 0; t < TN; ++t) b[kk][t] = *reinterpret_cast<const fbf16x8*>(lb + t * 2048 + (at ^ (32 * kk)));
        }
    };
    // The next stage has landed for all waves, two later ones are in flight; all LDS reads before are done.  (Beyond the end
    // copies that carry nothing are started, so that their number is the same everywhere: with branches around them the
    // compiler cannot tell which have landed and waits for all of them before it reads a stage.)
    auto land = [&] {
        fb_wait<2 * LD>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fb_barrier();
    };
    res_each<3>([&](auto N) { issue(decltype(N)::value, slot(N)); });
    land();
    issue(3, slot(std::integral_constant<int, 3>{}));
    read(std::integral_constant<int, 0>{}, fa[0], fb[0]);
    for (int s4 = 0; s4 < steps; s4 += 4)
        res_each<4>([&](auto N) {
            constexpr int v = decltype(N)::value;
            land();
            issue(s4 + v + 4, slot(N));
            __builtin_amdgcn_sched_barrier(0);
            read(std::integral_constant<int, v + 1>{}, fa[(v + 1) & 1], fb[(v + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int t = 0; t < TN; ++t) acc[m][t] = res_mma(fb[v & 1][kk][t], fa[v & 1][kk][m], acc[m][t]);
            __builtin_amdgcn_sched_barrier(0);
        });
    fb_wait<0>();   // no copy is in flight when the block ends
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            uint32_t o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = pack_bf16(acc[m][t][2 * e], acc[m][t][2 * e + 1]);
            res_store<false>(Out, co, r0 + 64 * wm + 32 * m, n, 32 * (TN * wn + t), co, o);
        }
}

// H, dG and dU of a tile of 128 rows by 64 hidden columns.
__global__ void __launch_bounds__(256, 2)
k_ffn_mid_bf16(const uint16_t* __restrict__ X, int64_t ldx, const uint16_t* __restrict__ dY, int64_t ldy, int64_t n, int ci,
               int co, const uint16_t* __restrict__ Wg, const uint16_t* __restrict__ Wu, int64_t ldw,
               const uint16_t* __restrict__ Wd, int64_t ldd, int f, int act, RowMat<uint16_t> H, RowMat<uint16_t> dG,
               RowMat<uint16_t> dU, int nf) {
    constexpr int MT = 4;
    typedef FbShape<2, 2, MT, 4> S;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::LDS];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nf * S::BM;
    const int c0 = (int)(u % nf) * 64, wave = threadIdx.x >> 6;
    floatx4 acc[MT][4], dh[MT][2];
    zero_acc(acc);
    zero_acc(dh);
    fb_product<2, 2, MT, 4, FB_KC, FB_MC, true>({row_major(X + r0 * ldx, ldx), n - r0}, {row_major(Wg + c0, ldw), f - c0},
                                                Wu + c0, ci, lds, acc);
    fb_barrier();
    fb_product<2, 2, MT, 2, FB_KC, FB_KC>({row_major(dY + r0 * ldy, ldy), n - r0},
                                          {row_major(Wd + (int64_t)c0 * ldd, ldd), f - c0}, nullptr, co, lds, dh);
    store_mid(acc, dh, r0 + 16 * MT * (wave >> 1), c0 + 32 * (wave & 1), n, act, H, dG, dU);
}

template <int WM, int WN, int MT, FbLay AL, FbLay BL>
__device__ __forceinline__ void dw_tile(const DwSide<uint16_t>& p, int t, int64_t r0, int64_t rows, uint8_t* lds,
                                        float* __restrict__ part) {
    typedef FbShape<WM, WN, MT, 4> S;
    const int m0 = t / p.tn * S::BM, c0 = t % p.tn * S::BN, wave = threadIdx.x >> 6;
    floatx4 acc[MT][4];
    zero_acc(acc);
    fb_product<WM, WN, MT, 4, AL, BL>({p.A.at(r0, m0), p.m - m0}, {p.B.at(r0, c0), p.nn - c0}, nullptr, rows, lds, acc);
    store_tile(acc, m0 + 16 * MT * (wave / WN), c0 + 64 * (wave % WN), p.m, p.nn, part + p.part, p.nn);
}

// Partial sums of both products over the rows of a chunk: the first in tiles of 16 MT0 x 256 (its rows are the
// channels), the second in tiles of 256 x 128 or, NARROW, 256 x 64 (its columns are).
template <int MT0, bool NARROW>
__global__ void __launch_bounds__(256, 2)
k_ffn_dw_bf16(DwSide<uint16_t> p0, DwSide<uint16_t> p1, int64_t n, int64_t chunk, int64_t per_chunk,
              float* __restrict__ part) {
    constexpr int MT1 = NARROW ? 4 : 8, WM1 = NARROW ? 4 : 2, WN1 = NARROW ? 1 : 2;
    typedef FbShape<1, 4, MT0, 4> S0;
    typedef FbShape<WM1, WN1, MT1, 4> S1;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S0::LDS > S1::LDS ? S0::LDS : S1::LDS];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int tiles = p0.tiles + p1.tiles;
    const int64_t s = u / tiles;
    const int t = (int)(u - s * tiles);
    const int64_t r0 = s * chunk, rows = n - r0 < chunk ? n - r0 : chunk;
    float* out = part + s * per_chunk;
    if (t < p0.tiles) dw_tile<1, 4, MT0, FB_MC, FB_MB>(p0, t, r0, rows, lds, out);
    else dw_tile<WM1, WN1, MT1, FB_MB, FB_MC>(p1, t - p0.tiles, r0, rows, lds, out);
}

// The weights' gradients from the chunks' sums, added in chunk order: per chunk dWg | dWu as ci x 2 fp, then dWd.
template <typename T>
__global__ void __launch_bounds__(kFfnThreads)
k_ffn_dw_sum(const float* __restrict__ part, int64_t chunks, int64_t per_chunk, int ci, int f, int fp, int co,
             T* __restrict__ dWg, T* __restrict__ dWu, T* __restrict__ dWd, int64_t up, int64_t total) {
    for (int64_t i = (int64_t)blockIdx.x * kFfnThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kFfnThreads) {
        T* out;
        if (i < up) {
            const int64_t row = i / (2 * fp);
            int col = (int)(i - row * 2 * fp);
            out = dWg;
            if (col >= fp) {
                out = dWu;
                col -= fp;
            }
            if (!out || col >= f) continue;
            out += row * f + col;
        } else {
            out = dWd + (i - up);
        }
        float s = 0.f;
#pragma unroll 4
        for (int64_t k = 0; k < chunks; ++k) s += part[k * per_chunk + i];
        store_out(out, s);
    }
}

// A few rows (at most R): out (n x nn) = A B, or act(A B) * (A B2) with B2.  Bound: the latency of one round of loads and of
// the sum over a block.  A thread takes 16 bytes of columns of every (threads / 4)-th reduction element, a block 4 x 16 bytes
// of columns, so that even a narrow layer is spread over many blocks and a thread has few elements.  The lanes' sums are
// added by halves (each lane passes on half of its values, then a quarter, ...): a quarter of the exchanges of adding every
// value over all lanes.
constexpr int kFewCols = 4;

template <int R>
constexpr int few_threads() { return R < 4 ? 1024 : 512; }   // (the registers of four rows' sums allow no more)

// v[0 .. N) summed over the lanes that differ in the bits of DIST, DIST / 2, ..., kFewCols; on return each lane holds the sums
// of N / (their number) values (at least one) in v[0 ..], from value `first` on.
template <int N, int DIST>
__device__ __forceinline__ void few_reduce(float* v, int& first) {
    if constexpr (DIST >= kFewCols) {
        const bool up = threadIdx.x & DIST;
        if constexpr (N > 1) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float send = up ? v[i] : v[i + N / 2], keep = up ? v[i + N / 2] : v[i];
                v[i] = keep + __shfl_xor(send, DIST, 64);
            }
            first += up ? N / 2 : 0;
            few_reduce<N / 2, DIST / 2>(v, first);
        } else {
            v[0] += __shfl_xor(v[0], DIST, 64);
            few_reduce<1, DIST / 2>(v, first);
        }
    }
}

template <typename TA, typename T, typename TO, int R, bool GATED>
__global__ void __launch_bounds__(few_threads<R>())
k_ffn_few(const TA* __restrict__ A, int64_t lda, int n, int k, const T* __restrict__ B, const T* __restrict__ B2, int nn,
          int act, TO* __restrict__ out, int64_t ldo) {
    typedef RowVec<T> RV;
    constexpr int V = RV::V, NB = GATED ? 2 : 1, N = NB * R * V, THREADS = few_threads<R>(), LANES = THREADS / kFewCols;
    constexpr int KEEP = N > 16 ? N / 16 : 1;   // values of a lane after the sum over its wave's 16 reduction lanes
    __shared__ float red[THREADS / 64][N * kFewCols];
    const int cl = threadIdx.x % kFewCols, kl = threadIdx.x / kFewCols;
    const int col = (blockIdx.x * kFewCols + cl) * V;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll 4
    for (int j = kl; j < k; j += LANES) {
        typename RV::Raw w[NB];
        w[0] = load_vec<T, true>(B + (int64_t)j * nn + col, nn - col);
        if (GATED) w[NB - 1] = load_vec<T, true>(B2 + (int64_t)j * nn + col, nn - col);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float a = r < n ? to_f32(A[r * lda + j]) : 0.f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[(b * R + r) * V + e] = fmaf(a, RV::get(w[b], e), acc[(b * R + r) * V + e]);
        }
    }
    int first = 0;
    few_reduce<N, 32>(acc, first);
    const int wave = threadIdx.x >> 6;
    // (with fewer values than lanes several lanes hold the same sum)
#pragma unroll
    for (int i = 0; i < KEEP; ++i) red[wave][(first + i) * kFewCols + cl] = acc[i];
    __syncthreads();
    for (int i = threadIdx.x; i < R * kFewCols * V; i += THREADS) {
        const int r = i / (kFewCols * V), c4 = i / V % kFewCols, e = i % V, c = (blockIdx.x * kFewCols + c4) * V + e;
        float v[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v[b] = 0.f;
            for (int w = 0; w < THREADS / 64; ++w) v[b] += red[w][((b * R + r) * V + e) * kFewCols + c4];
        }
        if (r >= n || c >= nn) continue;
        float o = v[0];
        if (GATED)
            with_act(act, [&](auto ACT) {
                float a, d;
                ffn_act<decltype(ACT)::value, false, sizeof(T) == 2>(v[0], a, d);
                o = a * v[NB - 1];
            });
        store_out(&out[r * ldo + c], o);
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static int64_t pad8(int64_t v) { return (v + 7) / 8 * 8; }
static size_t ffn_al256(size_t b) { return (b + 255) & ~(size_t)255; }

static bool ffn_sizes_ok(int32_t dtype, int64_t n, int32_t ci, int32_t f, int32_t co) {
    return (dtype == GSC_F32 || dtype == GSC_BF16) && n >= 0 && ci >= 1 && f >= 1 && co >= 1 && ci <= kFfnMaxWidth &&
           f <= kFfnMaxWidth && co <= kFfnMaxWidth && n <= ((int64_t)1 << 31) * 16;
}

struct FfnShape {
    int64_t n;
    int ci, f, co;
    int64_t fp;   // hidden columns in whole tiles
    FfnShape(int64_t n, int ci, int f, int co) : n(n), ci(ci), f(f), co(co), fp(ceil_div(f, 64) * 64) {}
};

// Workspace, in order: what the padded copies of X, dY (backward), Wg, Wu and Wd and the packed weights take
// (bfloat16), H, then for the backward pass dG | dU and the weight gradients' partial sums; each only where the kernels
// that take the call use it.  (The copies also for widths that need none: a call's addresses may.)
struct FfnLayout {
    bool few, res;      // k_ffn_few; rows in registers
    size_t x, dy, wg, wu, wd, pack, h, dgu, part, total;
    int64_t per_chunk, up, chunks, chunk;
    bool m_nar, n_nar;      // tiles of 64 channels for the weight gradients of the first, of the second projection
    int tn0, t0, tn1, t1;
};

// Whether tiles of 128 rows leave at most a quarter of their last round of compute units idle.
static bool ffn_fills(int64_t n) {
    const int64_t tiles = ceil_div(n, 128), cus = device_cus();
    return 4 * tiles >= 3 * ceil_div(tiles, cus) * cus;
}

// Whether the kernels that keep rows in registers can take a bfloat16 call at all.
static bool ffn_res_can(const FfnShape& d) { return d.ci <= kResMax && d.co <= kResMax; }

// ... and do.  Forward, up to 64 channels: from 40 tiles of 128 rows on (64 channels, 1,024 hidden: 4,000 rows 23.0 us, tiles
// 21.6; 6,000 rows 23.0 and 23.3; 12,000 rows 23.0 and 27.8; 256 hidden: 4,000 rows 10.8 and 10.9, 12,000 rows 10.9 and 12.0;
// 32 channels alike, 8 and 16 no difference).  Up to 128 channels: from 100 tiles on (128 channels, 512 hidden: 10,000 rows
// 19.0 and 17.8, 14,000 rows 19.2 and 20.6; 96 channels: 10,000 rows 15.0 and 14.4, 14,000 rows 15.2 and 16.0).  Wider ones
// take a block a compute unit: where they fill their rounds (256 channels: 30,000 rows 57 and 62 us, 45,000 rows in a second
// round of 96 blocks 98 and 87, 60,000 rows 105 and 119).
static bool ffn_res_fwd(const FfnShape& d) {
    if (!ffn_res_can(d)) return false;
    const int c = d.ci > d.co ? d.ci : d.co;
    return c > 128 ? ffn_fills(d.n) : ceil_div(d.n, 128) >= (c > 64 ? 100 : 40);
}
// Backward: once H, dG and dU outgrow the 256 MB of the last-level cache, where the tiles' traffic costs more than their better
// spread over the device saves (128 channels, 512 hidden: 60,000 rows 159 us, tiles 152; 90,000 rows 222 and 232; 200,000
// rows 477 and 520; 256 channels, 1,024 hidden: 30,000 rows 192 and 199, 90,000 rows 521 and 584), and not for 64 channels or
// less (forward and backward of 200,000 rows of 64: 221 and 215, with a kernel for them that is not here any more).
static bool ffn_res_bwd(const FfnShape& d) {
    return ffn_res_can(d) && (d.ci > 64 || d.co > 64) && d.n * d.fp * 6 >= (int64_t)256 << 20;
}

// float32: where the blocks fill their rounds (64 channels, 256 hidden, forward 16,000 rows 31 us, tiles 26; 32,000 rows 32
// and 41; 60,000 rows 55 and 70; backward 89 and 71, 110 and 116, 172 and 187, but 45,000 rows 162 and 150).  Forward of up
// to 32 channels, of which a compute unit takes several blocks: up to 128 hidden columns always (300 to 8,000 rows 10.5 to
// 10.8 us, tiles 10.8 to 11.2; 45,000 rows 18 and 25), more of them, which a block walks over one chunk after the other, from
// 150 tiles on (256 hidden: 1,000 rows 18.6 us, tiles 13.1, 16,000 rows 18.9 and 20.3, 24,000 rows 19.5 and 27.8; 1,024
// hidden: 65 and 33, 68 and 59, 67 and 86; 45,000 rows 111 and 136).
static bool ffn_res_f32(const FfnShape& d, bool bwd) {
    if (d.ci > kResMaxF32 || d.co > kResMaxF32) return false;
    return ffn_fills(d.n) || (!bwd && d.ci <= 32 && d.co <= 32 && (d.f <= 128 || ceil_div(d.n, 128) >= 150));
}

// Which of the two ways a call of either type and pass goes.
static bool ffn_res(int dtype, const FfnShape& d, bool bwd) {
    if (dtype != GSC_BF16) return ffn_res_f32(d, bwd);
    return bwd ? ffn_res_bwd(d) : ffn_res_fwd(d);
}

// Whether every launch of a call has fewer than 2^32 threads, the most that one takes.  Rows in registers: 512 (float32:
// 256) threads for 128 rows.  Tiles: 256 for at least 128 rows (fewer only where few tiles are) by 64 columns.
static bool ffn_launches(int dtype, const FfnShape& d, bool bwd) {
    const int64_t tiles = ceil_div(d.n, 128);
    int64_t widest = d.f > d.co ? d.f : d.co;
    if (bwd && d.ci > widest) widest = d.ci;
    const int64_t threads = !bwd && ffn_res(dtype, d, bwd) ? tiles * (dtype == GSC_BF16 ? 512 : 256)
                                                           : tiles * ceil_div(widest, 64) * 256;
    return threads < (int64_t)1 << 32;
}

// float32: tiles of 64 outputs instead of 128 in a direction where they leave less of the last one empty.
static bool ffn_narrow(int64_t rows) { return ceil_div(rows, 64) % 2 == 1 && rows < 512; }

// Row chunks of the weights' gradients: as many as fill the device once with two blocks a compute unit (twice as many blocks:
// backward pass of 300,000 rows, 256 channels, 1,024 hidden bf16 1,633 us, 1,589; 30,000 rows 243 and 203), of at least 512
// rows, or 128 up to 32 chunks: few rows leave the device to few blocks, whose length is what counts, many rows pay for each
// chunk's sums (backward pass, 64 channels, 256 hidden float32: 1,000 rows 35 us in chunks of 128 and 52 of 512; bfloat16:
// 30,000 rows 51 and 45 us).
static int64_t ffn_chunks(int64_t n, int64_t tiles) {
    int64_t most = ceil_div(n, 128);
    if (most > 32) most = ceil_div(n, 512) > 32 ? ceil_div(n, 512) : 32;
    const int64_t c = 512 / tiles < most ? 512 / tiles : most;
    return c < 1 ? 1 : c;
}

static FfnLayout ffn_layout(int dtype, const FfnShape& d, bool bwd) {
    FfnLayout L{};
    const size_t size = dtype == GSC_BF16 ? 2 : 4;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t a = at;
        at += ffn_al256(bytes);
        return a;
    };
    const int64_t rows = d.n > 0 ? d.n : 1;
    L.few = !bwd && d.n <= kFfnFewRows;
    L.res = !L.few && ffn_res(dtype, d, bwd);
    if (dtype == GSC_BF16 && (bwd || !(L.few || L.res))) {
        L.x = take((size_t)d.n * pad8(d.ci) * 2);
        if (bwd) L.dy = take((size_t)d.n * pad8(d.co) * 2);
        L.wg = take((size_t)d.ci * pad8(d.f) * 2);
        L.wu = take((size_t)d.ci * pad8(d.f) * 2);
        if (!L.res) L.wd = take((size_t)d.f * pad8(d.co) * 2);
    }
    if (dtype == GSC_BF16 && L.res) L.pack = take(res_pack_bytes(d.ci, d.f, d.co));
    const int64_t tiles = ceil_div(d.n, 128);
    if (L.few) L.h = take((size_t)d.n * 4 * d.fp);
    else if (bwd || !L.res) L.h = take((size_t)tiles * 128 * size * d.fp);
    if (bwd) {
        L.dgu = take((size_t)tiles * 128 * 2 * d.fp * size);
        int bm0, bn0, bm1, bn1;
        if (dtype == GSC_BF16) {
            L.m_nar = d.ci <= 64;
            L.n_nar = d.co <= 64;
            bm0 = L.m_nar ? 64 : 128;
            bn0 = bm1 = 256;
            bn1 = L.n_nar ? 64 : 128;
        } else {
            L.m_nar = ffn_narrow(d.ci);
            L.n_nar = ffn_narrow(d.co);
            bm0 = L.m_nar ? 64 : 128;
            bn0 = bm1 = 128;
            bn1 = L.n_nar ? 64 : 128;
        }
        L.tn0 = (int)ceil_div(2 * d.fp, bn0);
        L.t0 = (int)ceil_div(d.ci, bm0) * L.tn0;
        L.tn1 = (int)ceil_div(d.co, bn1);
        L.t1 = (int)ceil_div(d.f, bm1) * L.tn1;
        L.chunk = ceil_div(ceil_div(rows, ffn_chunks(d.n, (int64_t)L.t0 + L.t1)), 128) * 128;
        L.chunks = ceil_div(rows, L.chunk);
        L.up = (int64_t)d.ci * 2 * d.fp;
        L.per_chunk = L.up + (int64_t)d.f * d.co;
        L.part = take((size_t)L.chunks * L.per_chunk * sizeof(float));
    }
    L.total = at > 0 ? at : 256;
    return L;
}

// Row tiles of 64 (float32) or 128 (bfloat16) instead of twice as many where those would leave compute units idle.
static bool ffn_short(int64_t n, int rows, int64_t col_tiles) { return ceil_div(n, rows) * col_tiles < 2 * device_cus(); }

template <typename T>
static RowMat<const T> ffn_const(const RowMat<T>& m) { return {m.p, m.ld, m.gs, m.ts}; }

// --- float32
// f(WHOLE as a constant): the widths are multiples of four floats
template <typename F>
static void ffn_whole(const FfnShape& d, F f) {
    if (d.ci % 4 == 0 && d.f % 4 == 0 && d.co % 4 == 0) f(std::true_type{});
    else f(std::false_type{});
}

template <bool BKC, bool WHOLE>
static void ffn_gemm_f32(RowMat<const float> A1, RowMat<const float> A2, int64_t n, int64_t k, const float* B1,
                         const float* B2, int64_t ldb, int co, float* Out, hipStream_t s) {
    const bool nar = ffn_narrow(co);
    const int nc = (int)ceil_div(co, nar ? 64 : 128);
    const bool sho = ffn_short(n, 128, nc);
    auto* kern = sho ? (nar ? k_ffn_gemm_f32<BKC, 2, 2, WHOLE> : k_ffn_gemm_f32<BKC, 2, 4, WHOLE>)
                     : (nar ? k_ffn_gemm_f32<BKC, 4, 2, WHOLE> : k_ffn_gemm_f32<BKC, 4, 4, WHOLE>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(ceil_div(n, sho ? 64 : 128) * nc)), dim3(kFfnThreads), 0, s, A1, A2, n, k,
                       B1, B2, ldb, co, Out, nc);
}

static void ffn_fwd(const FfnShape& d, const FfnLayout& L, const float* X, const float* Wg, const float* Wu,
                    const float* Wd, int act, float* Y, char* ws, hipStream_t s) {
    if (L.res) return res_fwd(X, d.n, d.ci, Wg, Wu, d.f, Wd, d.co, act, Y, s);
    const RowMat<float> H = row_blocks(reinterpret_cast<float*>(ws + L.h), d.fp);
    const int nf = (int)ceil_div(d.f, 64);
    const bool sho = ffn_short(d.n, 128, nf);
    ffn_whole(d, [&](auto WHOLE) {
        constexpr bool W = decltype(WHOLE)::value;
        auto* up = sho ? k_ffn_up_f32<2, W> : k_ffn_up_f32<4, W>;
        hipLaunchKernelGGL(up, dim3((unsigned)(ceil_div(d.n, sho ? 64 : 128) * nf)), dim3(kFfnThreads), 0, s, X, d.n, d.ci,
                           Wg, Wu, d.f, act, H, nf);
        ffn_gemm_f32<false, W>(ffn_const(H), {}, d.n, d.f, Wd, nullptr, d.co, d.co, Y, s);
    });
}

static void ffn_bwd_rows(const FfnShape& d, const FfnLayout& L, const float* X, const float* Wg, const float* Wu,
                         const float* Wd, const float* dY, int act, float* dX, RowMat<float> H, RowMat<float> dG,
                         RowMat<float> dU, hipStream_t s) {
    if (L.res) return res_bwd(X, dY, d.n, d.ci, Wg, Wu, d.f, Wd, d.co, act, (int)d.fp, H, dG, dU, dX, s);
    const int nf = (int)ceil_div(d.f, 64);
    const bool sho = ffn_short(d.n, 128, nf);
    ffn_whole(d, [&](auto WHOLE) {
        constexpr bool W = decltype(WHOLE)::value;
        auto* mid = sho ? k_ffn_mid_f32<2, W> : k_ffn_mid_f32<4, W>;
        hipLaunchKernelGGL(mid, dim3((unsigned)(ceil_div(d.n, sho ? 64 : 128) * nf)), dim3(kFfnThreads), 0, s, X, dY, d.n,
                           d.ci, d.co, Wg, Wu, Wd, d.f, act, H, dG, dU, nf);
        if (dX) ffn_gemm_f32<true, W>(ffn_const(dG), ffn_const(dU), d.n, d.f, Wg, Wu, d.f, d.ci, dX, s);
    });
}

static void ffn_dw(const FfnShape& d, const FfnLayout& L, const DwSide<float>& p0, const DwSide<float>& p1, float* part,
                   hipStream_t s) {
    ffn_whole(d, [&](auto WHOLE) {
        constexpr bool W = decltype(WHOLE)::value;
        auto* kern = L.m_nar ? (L.n_nar ? k_ffn_dw_f32<2, 2, W> : k_ffn_dw_f32<2, 4, W>)
                             : (L.n_nar ? k_ffn_dw_f32<4, 2, W> : k_ffn_dw_f32<4, 4, W>);
        hipLaunchKernelGGL(kern, dim3((unsigned)(L.chunks * (p0.tiles + p1.tiles))), dim3(kFfnThreads), 0, s, p0, p1, d.n,
                           L.chunk, L.per_chunk, part);
    });
}

// --- bfloat16
// A matrix as the tiles take it: itself, or (whole) a padded copy that `pad` is to make.
struct FfnMat {
    const uint16_t* p;
    int64_t ld;
};
static FfnMat ffn_mat(const uint16_t* p, int64_t rows, int cols, char* copy, FfnPad& pad) {
    if (cols % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0) return {p, cols};
    const int i = pad.count++;
    pad.src[i] = p;
    pad.dst[i] = reinterpret_cast<uint16_t*>(copy);
    pad.cols[i] = cols;
    pad.ld[i] = (int)pad8(cols);
    pad.end[i] = (i ? pad.end[i - 1] : 0) + rows * (pad.ld[i] / 8);
    return {pad.dst[i], pad.ld[i]};
}
static void ffn_pad(const FfnPad& pad, hipStream_t s) {
    if (pad.count == 0) return;
    const int64_t blocks = ceil_div(pad.end[pad.count - 1], kFfnThreads);
    hipLaunchKernelGGL(k_ffn_pad, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kFfnThreads), 0, s, pad);
}

template <FbLay BL>
static void ffn_gemm_bf16(RowMat<const uint16_t> A1, RowMat<const uint16_t> A2, int64_t n, int64_t k, const uint16_t* B1,
                          const uint16_t* B2, int64_t ldb, int co, uint16_t* Out, hipStream_t s) {
    const bool nar = co <= 64;
    const int nc = (int)ceil_div(co, nar ? 64 : 128);
    const bool sho = !nar && ffn_short(n, 256, nc);
    auto* kern = nar ? k_ffn_gemm_bf16<4, 1, 4, BL> : (sho ? k_ffn_gemm_bf16<2, 2, 4, BL> : k_ffn_gemm_bf16<2, 2, 8, BL>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(ceil_div(n, sho ? 128 : 256) * nc)), dim3(256), 0, s, A1, A2, n, k, B1, B2, ldb,
                       co, Out, nc);
}

static void ffn_fwd(const FfnShape& d, const FfnLayout& L, const uint16_t* X, const uint16_t* Wg, const uint16_t* Wu,
                    const uint16_t* Wd, int act, uint16_t* Y, char* ws, hipStream_t s) {
    if (L.res) return res_fwd(X, d.n, d.ci, Wg, Wu, d.f, Wd, d.co, act, Y, ws + L.pack, s);
    const RowMat<uint16_t> H = row_blocks(reinterpret_cast<uint16_t*>(ws + L.h), d.fp);
    FfnPad pad{};
    const FfnMat x = ffn_mat(X, d.n, d.ci, ws + L.x, pad), g = ffn_mat(Wg, d.ci, d.f, ws + L.wg, pad),
                 u = ffn_mat(Wu, d.ci, d.f, ws + L.wu, pad), w = ffn_mat(Wd, d.f, d.co, ws + L.wd, pad);
    ffn_pad(pad, s);
    const int nf = (int)ceil_div(d.f, 64);
    const bool sho = ffn_short(d.n, 256, nf);
    auto* up = sho ? k_ffn_up_bf16<4> : k_ffn_up_bf16<8>;
    hipLaunchKernelGGL(up, dim3((unsigned)(ceil_div(d.n, sho ? 128 : 256) * nf)), dim3(256), 0, s, x.p, x.ld, d.n, d.ci,
                       g.p, u.p, g.ld, d.f, act, H, nf);
    ffn_gemm_bf16<FB_MC>(ffn_const(H), {}, d.n, d.f, w.p, nullptr, w.ld, d.co, Y, s);
}

static void ffn_dw(const FfnShape& d, const FfnLayout& L, const DwSide<uint16_t>& p0, const DwSide<uint16_t>& p1, float* part,
                   hipStream_t s) {
    auto* kern = L.m_nar ? (L.n_nar ? k_ffn_dw_bf16<4, true> : k_ffn_dw_bf16<4, false>)
                         : (L.n_nar ? k_ffn_dw_bf16<8, true> : k_ffn_dw_bf16<8, false>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(L.chunks * (p0.tiles + p1.tiles))), dim3(256), 0, s, p0, p1, d.n, L.chunk,
                       L.per_chunk, part);
}

// Tiles of 256 x 256, a block a compute unit, for one tile of columns that is more than half full, at least 768 hidden columns
// (less, and filling the pipeline costs what the shared operands save) and blocks that fill an eighth less than
// whole rounds of the device or more.  dH, dG, dU and dX of 256 channels, 64 outputs, such tiles and the others: 1,024 hidden
// 60,000 rows 242 and 272 us, 300,000 1,070 and 1,080, but 90,000 rows (1.4 rounds) 345 and 338, 33,000 (half a round) 125 and
// 128 (160 channels 109 and 104); 512 hidden 300,000 rows 597 and 589.  Two tiles of columns: 264 channels, 60,000 rows, 1,024
// hidden 296 and 291, 300,000 rows 1,450 and 1,339; 512 channels 356 and 367, 1,748 and 1,728.  128 channels: no difference.
static bool ffn_dx_wide(int64_t n, int64_t f, int ci) {
    const int64_t blocks = ceil_div(n, 256), cus = device_cus();
    return ci > 128 && ci <= 256 && f >= 768 && 8 * blocks >= 7 * ceil_div(blocks, cus) * cus;
}
static void ffn_dx_bf16(RowMat<const uint16_t> dG, RowMat<const uint16_t> dU, int64_t n, int64_t f, const uint16_t* Wg,
                        const uint16_t* Wu, int64_t ldw, int ci, uint16_t* dX, hipStream_t s) {
    if (!ffn_dx_wide(n, f, ci)) return ffn_gemm_bf16<FB_KC>(dG, dU, n, f, Wg, Wu, ldw, ci, dX, s);
    hipLaunchKernelGGL(k_ffn_gemm_kc, dim3((unsigned)ceil_div(n, 256)), dim3(512), 0, s, dG, dU, n, f, Wg, Wu, ldw, ci, dX);
}

// --- either type
// A few rows: H in float32 (no matrix core takes it, and it stays in the L2).
template <typename T>
static void ffn_fwd_few(const FfnShape& d, const FfnLayout& L, const T* X, const T* Wg, const T* Wu, const T* Wd, int act,
                        T* Y, char* ws, hipStream_t s) {
    constexpr int W = kFewCols * (16 / (int)sizeof(T));
    float* H = reinterpret_cast<float*>(ws + L.h);
    const int n = (int)d.n;
    auto* up = n == 1 ? k_ffn_few<T, T, float, 1, true>
                      : (n == 2 ? k_ffn_few<T, T, float, 2, true> : k_ffn_few<T, T, float, 4, true>);
    auto* down = n == 1 ? k_ffn_few<float, T, T, 1, false>
                        : (n == 2 ? k_ffn_few<float, T, T, 2, false> : k_ffn_few<float, T, T, 4, false>);
    const int threads = n <= 2 ? few_threads<1>() : few_threads<4>();
    hipLaunchKernelGGL(up, dim3((unsigned)ceil_div(d.f, W)), dim3(threads), 0, s, X, (int64_t)d.ci, n, d.ci, Wg, Wu, d.f, act,
                       H, d.fp);
    hipLaunchKernelGGL(down, dim3((unsigned)ceil_div(d.co, W)), dim3(threads), 0, s, (const float*)H, d.fp, n, d.f, Wd,
                       (const T*)nullptr, d.co, act, Y, (int64_t)d.co);
}

template <typename T>
static void ffn_bwd(const FfnShape& d, const FfnLayout& L, const T* X, const T* Wg, const T* Wu, const T* Wd, const T* dY,
                    int act, T* dX, T* dWg, T* dWu, T* dWd, char* ws, hipStream_t s) {
    const int64_t n = d.n;
    // dG and dU share their blocks of 128 rows: the gradients of both projections are one product with X
    const RowMat<T> H = row_blocks(reinterpret_cast<T*>(ws + L.h), d.fp),
                    dG = row_blocks(reinterpret_cast<T*>(ws + L.dgu), 2 * d.fp), dU = dG.at(0, d.fp);
    float* part = reinterpret_cast<float*>(ws + L.part);
    const T *xs = X, *ys = dY;
    int64_t ldx = d.ci, ldy = d.co;
    if (n > 0) {
        if constexpr (sizeof(T) == 2) {
            FfnPad pad{};
            const FfnMat x = ffn_mat(X, n, d.ci, ws + L.x, pad), y = ffn_mat(dY, n, d.co, ws + L.dy, pad),
                         g = ffn_mat(Wg, d.ci, d.f, ws + L.wg, pad), u = ffn_mat(Wu, d.ci, d.f, ws + L.wu, pad),
                         w = L.res ? FfnMat{} : ffn_mat(Wd, d.f, d.co, ws + L.wd, pad);
            ffn_pad(pad, s);
            xs = x.p;
            ys = y.p;
            ldx = x.ld;
            ldy = y.ld;
            const int nf = (int)ceil_div(d.f, 64);
            if (L.res) {
                res_mid(X, dY, n, d.ci, Wg, Wu, d.f, Wd, d.co, act, H, dG, dU, ws + L.pack, s);
            } else {
                hipLaunchKernelGGL(k_ffn_mid_bf16, dim3((unsigned)(ceil_div(n, 128) * nf)), dim3(256), 0, s, x.p, x.ld,
                                   y.p, y.ld, n, d.ci, d.co, g.p, u.p, g.ld, w.p, w.ld, d.f, act, H, dG, dU, nf);
            }
            if (dX) ffn_dx_bf16(ffn_const(dG), ffn_const(dU), n, d.f, g.p, u.p, g.ld, d.ci, dX, s);
        } else {
            ffn_bwd_rows(d, L, X, Wg, Wu, Wd, dY, act, dX, H, dG, dU, s);
        }
    }
    if (!dWg && !dWu && !dWd) return;
    const bool up = dWg || dWu;
    const DwSide<T> p0{row_major(xs, ldx), ffn_const(dG), d.ci, (int)(2 * d.fp), L.tn0, up ? L.t0 : 0, 0};
    const DwSide<T> p1{ffn_const(H), row_major(ys, ldy), d.f, d.co, L.tn1, dWd ? L.t1 : 0, L.up};
    if (n > 0) ffn_dw(d, L, p0, p1, part, s);
    const int64_t total = dWd ? L.per_chunk : L.up;
    const int64_t blocks = ceil_div(total, kFfnThreads);
    hipLaunchKernelGGL(k_ffn_dw_sum<T>, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kFfnThreads), 0, s, part,
                       n > 0 ? L.chunks : 0, L.per_chunk, d.ci, d.f, (int)d.fp, d.co, dWg, dWu, dWd, L.up, total);
}

}  // namespace gsc

using namespace gsc;

extern "C" {

size_t gsc_gated_ffn_fwd_ws_bytes(int32_t dtype, int64_t n, int32_t c_in, int32_t hidden, int32_t c_out) {
    if (!ffn_sizes_ok(dtype, n, c_in, hidden, c_out)) return 0;
    return ffn_layout(dtype, FfnShape(n, c_in, hidden, c_out), false).total;
}

int gsc_gated_ffn_fwd(int32_t dtype, const void* X, int64_t n, int32_t c_in, const void* Wg, const void* Wu,
                      int32_t hidden, const void* Wd, int32_t c_out, int32_t act, void* Y, void* ws, size_t ws_bytes,
                      void* stream) {
    clear_error();
    if (dtype != GSC_F32 && dtype != GSC_BF16) return fail(GSC_EINVAL, "gated_ffn_fwd: unknown dtype %d", dtype);
    if (act < GSC_GATE_SILU || act > GSC_GATE_SIGMOID) return fail(GSC_EINVAL, "gated_ffn_fwd: unknown act %d", act);
    if (!ffn_sizes_ok(dtype, n, c_in, hidden, c_out))
        return fail(GSC_EINVAL, "gated_ffn_fwd: bad sizes n=%lld c_in=%d hidden=%d c_out=%d", (long long)n, c_in, hidden,
                    c_out);
    const FfnShape d(n, c_in, hidden, c_out);
    if (!ffn_launches(dtype, d, false)) return fail(GSC_EINVAL, "gated_ffn_fwd: more rows and columns than a launch takes");
    if (n == 0) return GSC_OK;
    if (!X || !Wg || !Wu || !Wd || !Y) return fail(GSC_EINVAL, "gated_ffn_fwd: null X/Wg/Wu/Wd/Y");
    const FfnLayout L = ffn_layout(dtype, d, false);
    if (!ws || ws_bytes < L.total)
        return fail(GSC_ESHORT, "gated_ffn_fwd: ws needs %zu bytes, got %zu", L.total, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(GSC_EINVAL, "gated_ffn_fwd: ws must be aligned to 16 bytes");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    auto run = [&](auto t) {
        typedef decltype(t) T;
        const T *x = (const T*)X, *g = (const T*)Wg, *u = (const T*)Wu, *w = (const T*)Wd;
        if (L.few) ffn_fwd_few<T>(d, L, x, g, u, w, act, (T*)Y, (char*)ws, s);
        else ffn_fwd(d, L, x, g, u, w, act, (T*)Y, (char*)ws, s);
    };
    if (dtype == GSC_BF16) run(uint16_t{});
    else run(float{});
    GSC_LAUNCH_CHECK();
    return GSC_OK;
}

size_t gsc_gated_ffn_bwd_ws_bytes(int32_t dtype, int64_t n, int32_t c_in, int32_t hidden, int32_t c_out) {
    if (!ffn_sizes_ok(dtype, n, c_in, hidden, c_out)) return 0;
    return ffn_layout(dtype, FfnShape(n, c_in, hidden, c_out), true).total;
}

int gsc_gated_ffn_bwd(int32_t dtype, const void* X, int64_t n, int32_t c_in, const void* Wg, const void* Wu,
                      int32_t hidden, const void* Wd, int32_t c_out, const void* dY, int32_t act, void* dX, void* dWg,
                      void* dWu, void* dWd, void* ws, size_t ws_bytes, void* stream) {
    clear_error();
    if (dtype != GSC_F32 && dtype != GSC_BF16) return fail(GSC_EINVAL, "gated_ffn_bwd: unknown dtype %d", dtype);
    if (act < GSC_GATE_SILU || act > GSC_GATE_SIGMOID) return fail(GSC_EINVAL, "gated_ffn_bwd: unknown act %d", act);
    if (!ffn_sizes_ok(dtype, n, c_in, hidden, c_out))
        return fail(GSC_EINVAL, "gated_ffn_bwd: bad sizes n=%lld c_in=%d hidden=%d c_out=%d", (long long)n, c_in, hidden,
                    c_out);
    const FfnShape d(n, c_in, hidden, c_out);
    if (!ffn_launches(dtype, d, true)) return fail(GSC_EINVAL, "gated_ffn_bwd: more rows and columns than a launch takes");
    if (!dX && !dWg && !dWu && !dWd) return GSC_OK;
    if (n == 0 && !dWg && !dWu && !dWd) return GSC_OK;
    if (n > 0 && (!X || !Wg || !Wu || !Wd || !dY)) return fail(GSC_EINVAL, "gated_ffn_bwd: null X/Wg/Wu/Wd/dY");
    const FfnLayout L = ffn_layout(dtype, d, true);
    if (!ws || ws_bytes < L.total)
        return fail(GSC_ESHORT, "gated_ffn_bwd: ws needs %zu bytes, got %zu", L.total, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(GSC_EINVAL, "gated_ffn_bwd: ws must be aligned to 16 bytes");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    auto run = [&](auto t) {
        typedef decltype(t) T;
        ffn_bwd<T>(d, L, (const T*)X, (const T*)Wg, (const T*)Wu, (const T*)Wd, (const T*)dY, act, (T*)dX, (T*)dWg,
                   (T*)dWu, (T*)dWd, (char*)ws, s);
    };
    if (dtype == GSC_BF16) run(uint16_t{});
    else run(float{});
    GSC_LAUNCH_CHECK();
    return GSC_OK;
}

}  // extern "C"
