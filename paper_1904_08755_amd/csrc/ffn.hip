// Gated feed-forward block of feature rows, forward and backward.
//
//   G = X Wg,  U = X Wu,  H = act(G) * U,  Y = H Wd
//   dH = dY Wd^T,  dG = dH U act'(G),  dU = dH act(G)
//   dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU,  dWd = H^T dY
//
// Products run on the matrix cores (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4f32) with float32
// sums.  The forward pass is two kernels: both projections with the activation and the product
// (k_ffn_up: G and U never leave the registers), then the output projection (k_ffn_gemm).  The
// backward pass works G and U out again from X (a third more products than reading them back, but the
// forward pass need not write them nor the program keep them: at 256 channels and 1,024 hidden
// ones their two arrays would be eight times the bytes of X): k_ffn_mid computes G, U and dH of a tile and
// stores H, dG and dU; k_ffn_gemm adds dX; k_ffn_dw adds the weights' gradients over row chunks and
// k_ffn_dw_sum adds the chunks in order, so that every result is bit-reproducible.
//
// bfloat16: G, U, dH and all sums stay in float32; H, dG and dU are rounded to bfloat16 once, as the
// matrix cores take them, and the results once as they are stored.
//
// One tile product serves all of them (tile_product): 32 MT x 32 NT outputs per block of four waves,
// the operands' next 128 bytes of the reduction in registers while the current ones are read from
// LDS (two stages, one barrier a step).  An operand lies either with the reduction along its rows
// (KC) or across them (MC); both are copied to LDS as they lie, and an MC operand's bfloat16 fragments
// are read with the LDS transpose read (ds_read_b64_tr_b16: within each 16 lanes, lane i receives
// element i % 4 of the 8-byte pieces that lanes i / 4, i / 4 + 4, i / 4 + 8, i / 4 + 12 address).
#include "row_vec.h"

namespace gsc {

constexpr int kFfnThreads = 256;
constexpr int kFfnRowBytes = 128;                       // reduction bytes of a step
constexpr int kFfnMaxWidth = 1 << 20;
constexpr int kFfnFewRows = 4;                          // rows up to which k_ffn_few runs

template <typename T>
constexpr int ffn_bk() { return kFfnRowBytes / (int)sizeof(T); }

typedef __bf16 fbf16x8 __attribute__((ext_vector_type(8)));
typedef short fs16x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// activations
// ---------------------------------------------------------------------------
__device__ __forceinline__ float ffn_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }
__device__ __forceinline__ float ffn_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + ffn_exp(-x)); }

// act(g) and (D) its derivative.  The hardware's exponential and reciprocal: within about |g| + 2 units in
// the last place of float32, far inside what the products' sums lose.
template <int ACT, bool D>
__device__ __forceinline__ void ffn_act(float g, float& a, float& d) {
    if constexpr (ACT == GSC_GATE_RELU) {
        a = g < 0.f ? 0.f : g;   // NaN passes through
        if (D) d = g > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == GSC_GATE_SIGMOID) {
        a = ffn_sigmoid(g);
        if (D) d = a * (1.f - a);
    } else if constexpr (ACT == GSC_GATE_SILU) {
        const float p = ffn_sigmoid(g);
        a = g * p;
        if (D) d = fmaf(a, 1.f - p, p);
    } else if constexpr (ACT == GSC_GATE_GELU) {
        // the normal distribution function from Abramowitz & Stegun 7.1.26 (absolute error of erf 1.5e-7),
        // its density shared with the derivative
        const float z = fabsf(g) * 0.70710678118655f;
        const float e = ffn_exp(-0.5f * g * g);
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
        float q = fmaf(1.061405429f, t, -1.453152027f);
        q = fmaf(q, t, 1.421413741f);
        q = fmaf(q, t, -0.284496736f);
        q = fmaf(q, t, 0.254829592f);
        q = 0.5f * q * t * e;              // the upper tail at |g|
        const float p = g < 0.f ? q : 1.f - q;
        a = g * p;
        if (D) d = fmaf(g * 0.398942280401433f, e, p);
    } else {
        // 0.5 (1 + tanh(u)) = sigmoid(2 u)
        const float k = 0.797884560802865f, c = 0.044715f;
        const float g2 = g * g;
        const float p = ffn_sigmoid(2.f * k * g * fmaf(c, g2, 1.f));
        a = g * p;
        if (D) d = fmaf(2.f * a * (1.f - p), k * fmaf(3.f * c, g2, 1.f), p);
    }
}

// f(activation as a constant)
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case GSC_GATE_RELU: f(std::integral_constant<int, GSC_GATE_RELU>{}); break;
        case GSC_GATE_SIGMOID: f(std::integral_constant<int, GSC_GATE_SIGMOID>{}); break;
        case GSC_GATE_GELU: f(std::integral_constant<int, GSC_GATE_GELU>{}); break;
        case GSC_GATE_GELU_TANH: f(std::integral_constant<int, GSC_GATE_GELU_TANH>{}); break;
        default: f(std::integral_constant<int, GSC_GATE_SILU>{}); break;
    }
}

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------
// One side of a product: `rows` outputs by k reduction elements, element (r, k) at p[r ld + k] (KC)
// or p[k ld + r] (MC).  Rows and reduction elements behind the end read as 0.  SPLIT: the tile's rows
// [0, R / 2) come from p and the others from p2 (both from row 0 on).
template <typename T>
struct Side {
    const T* p;
    const T* p2;
    int64_t ld;
    int64_t rows;
    int64_t k;
};

// A thread's share of a tile of R rows by one step, through registers into LDS.
template <typename T, bool KC, int R, bool SPLIT>
struct TileCopy {
    static constexpr int V = 16 / sizeof(T), BK = ffn_bk<T>();
    static constexpr int N = R * kFfnRowBytes / 16 / kFfnThreads;   // 16-byte pieces a thread
    static constexpr int PER = KC ? BK / V : R / V;                 // pieces of a row (KC) or of a reduction element
    static_assert(N >= 1 && kFfnThreads % PER == 0, "tile");
    typedef typename RowVec<T>::Raw Raw;

    const T* base;      // element (0, 0) of the thread's side
    int64_t ld;
    int line, at;       // first row (KC) or reduction element (MC), and the piece's first element across
    int64_t across;     // MC: elements from `at` to the rows' end
    int lim;            // KC: valid lines
    Raw r[N];

    __device__ __forceinline__ void start(const Side<T>& s) {
        const int c = threadIdx.x % PER;
        line = threadIdx.x / PER;
        at = c * V;
        base = s.p;
        ld = s.ld;
        if (KC) {
            lim = (int)(s.rows < R ? s.rows : R);
            across = 0;
        } else {
            int col = at;
            if (SPLIT && at >= R / 2) {
                base = s.p2;
                col -= R / 2;
            }
            across = s.rows - col;
            if (SPLIT && across > R / 2 - col) across = R / 2 - col;
            base += col;
            lim = 0;
        }
    }
    // the step at reduction element k0
    __device__ __forceinline__ void fetch(int64_t k0, int64_t k) {
        constexpr int DL = kFfnThreads / PER;   // lines between a thread's pieces
        if (KC) {
            const T* b = base + k0 + at;
            const int64_t left = k - k0 - at;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int row = line + j * DL;
                r[j] = load_vec<T, true>(b + (int64_t)row * ld, row < lim ? left : 0);
            }
        } else {
            const T* b = base + k0 * ld;
            const int kl = (int)(k - k0 < BK ? k - k0 : BK);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int kk = line + j * DL;
                r[j] = load_vec<T, true>(b + (int64_t)kk * ld, kk < kl ? across : 0);
            }
        }
    }
    __device__ __forceinline__ void put(uint8_t* lds) const {
        constexpr int DL = kFfnThreads / PER;
        const int c = threadIdx.x % PER;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = line + j * DL;
            *reinterpret_cast<uint4*>(lds + place(row, c)) = uint4{r[j][0], r[j][1], r[j][2], r[j][3]};
        }
    }
    // Byte of piece c of a line.  KC: lines of 128 bytes, pieces permuted by the row modulo 8, so the
    // eight rows that a read serves together lie in distinct banks.  MC bfloat16: 32-byte pairs of pieces
    // permuted by bits 0, 1 and 3 of the reduction element (the eight that a transpose read serves
    // together); float32: 64-byte groups permuted by bits 2 and 3.
    static __device__ __forceinline__ int place(int row, int c) {
        if (KC) return row * kFfnRowBytes + ((c ^ (row & 7)) * 16);
        if constexpr (sizeof(T) == 2) {
            constexpr int M = PER / 2 - 1;   // pairs of a line - 1
            return row * (R * 2) + (((c >> 1) ^ (((row & 3) | ((row >> 1) & 4)) & M)) * 32) + (c & 1) * 16;
        } else {
            constexpr int M = PER / 4 - 1;
            return row * (R * 4) + (((c >> 2) ^ ((row >> 2) & 3 & M)) * 64) + (c & 3) * 16;
        }
    }
};

// Fragment reads of one wave: operand of 16 rows from row0, reduction elements of group kk (32 of
// bfloat16, 16 of float32) of the step; lane (i, q) holds row i, elements 8 q .. 8 q + 7 (bfloat16)
// or 4 q .. 4 q + 3 (float32).
template <typename T, bool KC, int R>
struct Frag;
template <bool KC, int R>
struct Frag<uint16_t, KC, R> {
    typedef fbf16x8 Reg;
    static __device__ __forceinline__ Reg read(const uint8_t* lds, int row0, int kk) {
        const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
        if constexpr (KC) {
            const int row = row0 + i;
            return *reinterpret_cast<const fbf16x8*>(lds + row * kFfnRowBytes + (((kk * 4 + q) ^ (row & 7)) * 16));
        } else {
            // 8-byte piece i % 4 of the 16 rows, at reduction elements 8 q + i / 4 and four further
            const int k0 = kk * 32 + 8 * q + (i >> 2);
            constexpr int M = R / 16 - 1;
            const int x = ((k0 & 3) | ((k0 >> 1) & 4)) & M;
            const int at = k0 * (R * 2) + (((row0 >> 4) ^ x) * 32) + 8 * (i & 3);
            typedef __attribute__((address_space(3))) fs16x4* P;
            const fs16x4 v[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at)),
                                 __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at + 4 * R * 2))};
            return __builtin_bit_cast(fbf16x8, v);
        }
    }
    static __device__ __forceinline__ floatx4 mma(const Reg& a, const Reg& b, floatx4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <bool KC, int R>
struct Frag<float, KC, R> {
    typedef floatx4 Reg;
    static __device__ __forceinline__ Reg read(const uint8_t* lds, int row0, int kk) {
        const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
        if constexpr (KC) {
            const int row = row0 + i;
            return *reinterpret_cast<const floatx4*>(lds + row * kFfnRowBytes + (((kk * 4 + q) ^ (row & 7)) * 16));
        } else {
            constexpr int M = R / 16 - 1;
            floatx4 v;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k = kk * 16 + 4 * q + s;
                v[s] = *reinterpret_cast<const float*>(lds + k * (R * 4) + (((row0 >> 4) ^ (q & M)) * 64) + i * 4);
            }
            return v;
        }
    }
    static __device__ __forceinline__ floatx4 mma(const Reg& a, const Reg& b, floatx4 c) {
#pragma unroll
        for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], b[s], c, 0, 0, 0);
        return c;
    }
};

// LDS of a block: two stages of both operands.
template <int MT, int NT>
constexpr int ffn_lds() { return 2 * 32 * (MT + NT) * kFfnRowBytes; }

// acc[mi][ni] += the tile's product.  Four waves, (wm, wn) = 2 x 2: wave rows 16 MT wm .., columns
// 16 NT wn .. (SPLIT: half of them from either half of the tile's columns).  The second operand goes
// into the MFMA first, so lane (i, q) gets row 16 mi + i of its rows and four consecutive columns 4 q ..
// of block ni.  LDS may be in use by other waves' earlier reads: starts with a barrier.
template <typename T, bool AKC, bool BKC, int MT, int NT, bool SPLIT>
__device__ __forceinline__ void tile_product(const Side<T>& A, const Side<T>& B, uint8_t* lds, floatx4 (&acc)[MT][NT]) {
    constexpr int RA = 32 * MT, RB = 32 * NT, BK = ffn_bk<T>();
    constexpr int STAGE = (RA + RB) * kFfnRowBytes;
    typedef Frag<T, AKC, RA> FA;
    typedef Frag<T, BKC, RB> FB;
    TileCopy<T, AKC, RA, false> ca;
    TileCopy<T, BKC, RB, SPLIT> cb;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int64_t K = A.k;
    ca.start(A);
    cb.start(B);
    ca.fetch(0, K);
    cb.fetch(0, B.k);
    __syncthreads();
    ca.put(lds);
    cb.put(lds + RA * kFfnRowBytes);
    __syncthreads();
    int cur = 0;
    for (int64_t k0 = 0; k0 < K; k0 += BK) {
        const bool more = k0 + BK < K;
        if (more) {
            ca.fetch(k0 + BK, K);
            cb.fetch(k0 + BK, B.k);
        }
        const uint8_t* la = lds + cur * STAGE;
        const uint8_t* lb = la + RA * kFfnRowBytes;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            typename FA::Reg a[MT], b[NT];
#pragma unroll
            for (int mi = 0; mi < MT; ++mi) a[mi] = FA::read(la, 16 * (MT * wm + mi), kk);
#pragma unroll
            for (int ni = 0; ni < NT; ++ni) {
                const int col = !SPLIT ? 16 * (NT * wn + ni)
                                       : 16 * (NT / 2 * wn + ni % (NT / 2)) + (ni < NT / 2 ? 0 : RB / 2);
                b[ni] = FB::read(lb, col, kk);
            }
#pragma unroll
            for (int mi = 0; mi < MT; ++mi)
#pragma unroll
                for (int ni = 0; ni < NT; ++ni) acc[mi][ni] = FA::mma(b[ni], a[mi], acc[mi][ni]);
        }
        if (more) {
            cur ^= 1;
            uint8_t* ld = lds + cur * STAGE;
            ca.put(ld);
            cb.put(ld + RA * kFfnRowBytes);
        }
        __syncthreads();
    }
}

template <int MT, int NT>
__device__ __forceinline__ void zero_acc(floatx4 (&acc)[MT][NT]) {
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
}

// four consecutive columns of a row
__device__ __forceinline__ void store4(float* p, int64_t left, const float (&v)[4]) {
    if (left >= 4) {
        *reinterpret_cast<floatx4u*>(p) = floatx4u{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = v[e];
    }
}
__device__ __forceinline__ void store4(uint16_t* p, int64_t left, const float (&v)[4]) {
    typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));
    if (left >= 4) {
        *reinterpret_cast<u32x2u*>(p) = u32x2u{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) store_out(&p[e], v[e]);
    }
}

// ---------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------
// H (n x ldh, columns behind f zero) of a tile of 32 MT rows by 64 hidden columns.
template <typename T, int MT>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_up(const T* __restrict__ X, int64_t n, int ci, const T* __restrict__ Wg, const T* __restrict__ Wu, int f, int act,
         T* __restrict__ H, int64_t ldh, int nf) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, 4>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nf * (32 * MT);
    const int c0 = (int)(u % nf) * 64;
    floatx4 acc[MT][4];
    zero_acc(acc);
    tile_product<T, true, false, MT, 4, true>({X + r0 * ci, nullptr, ci, n - r0, ci},
                                              {Wg + c0, Wu + c0, f, f - c0, ci}, lds, acc);
    const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
    with_act(act, [&](auto ACT) {
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
            const int64_t row = r0 + 16 * (MT * wm + mi) + i;
            if (row >= n) continue;
#pragma unroll
            for (int ni = 0; ni < 2; ++ni) {
                const int col = c0 + 16 * (2 * wn + ni) + 4 * q;
                float h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, d;
                    ffn_act<decltype(ACT)::value, false>(acc[mi][ni][e], a, d);
                    h[e] = a * acc[mi][ni + 2][e];
                }
                store4(H + row * ldh + col, ldh - col, h);
            }
        }
    });
}

// Out (n x co) = A1 B1 (+ A2 B2 where A2 is given): A rows of the reduction (KC), B either way.
template <typename T, bool BKC, int MT, int NT>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_gemm(const T* __restrict__ A1, const T* __restrict__ A2, int64_t lda, int64_t n, int64_t ka,
           const T* __restrict__ B1, const T* __restrict__ B2, int64_t ldb, int64_t kb, int co, T* __restrict__ Out,
           int nc) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, NT>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nc * (32 * MT);
    const int c0 = (int)(u % nc) * (32 * NT);
    floatx4 acc[MT][NT];
    zero_acc(acc);
    for (int s = 0; s < 2; ++s) {
        const T* A = s ? A2 : A1;
        const T* B = s ? B2 : B1;
        if (!A) break;
        tile_product<T, true, BKC, MT, NT, false>(
            {A + r0 * lda, nullptr, lda, n - r0, ka},
            {BKC ? B + (int64_t)c0 * ldb : B + c0, nullptr, ldb, co - c0, kb}, lds, acc);
    }
    const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) {
        const int64_t row = r0 + 16 * (MT * wm + mi) + i;
        if (row >= n) continue;
#pragma unroll
        for (int ni = 0; ni < NT; ++ni) {
            const int col = c0 + 16 * (NT * wn + ni) + 4 * q;
            const float v[4] = {acc[mi][ni][0], acc[mi][ni][1], acc[mi][ni][2], acc[mi][ni][3]};
            if (col < co) store4(Out + row * co + col, co - col, v);
        }
    }
}

// H (n x f8) and dG, dU (n x 2 f8, side by side) of a tile of 32 MT rows by 64 hidden columns.
template <typename T, int MT>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_mid(const T* __restrict__ X, const T* __restrict__ dY, int64_t n, int ci, int co, const T* __restrict__ Wg,
          const T* __restrict__ Wu, const T* __restrict__ Wd, int f, int act, T* __restrict__ H, T* __restrict__ dGU,
          int f8, int nf) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, 4>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int64_t r0 = u / nf * (32 * MT);
    const int c0 = (int)(u % nf) * 64;
    floatx4 acc[MT][4], dh[MT][2];
    zero_acc(acc);
    zero_acc(dh);
    tile_product<T, true, false, MT, 4, true>({X + r0 * ci, nullptr, ci, n - r0, ci},
                                              {Wg + c0, Wu + c0, f, f - c0, ci}, lds, acc);
    tile_product<T, true, true, MT, 2, false>({dY + r0 * co, nullptr, co, n - r0, co},
                                              {Wd + (int64_t)c0 * co, nullptr, co, f - c0, co}, lds, dh);
    const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
    with_act(act, [&](auto ACT) {
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
            const int64_t row = r0 + 16 * (MT * wm + mi) + i;
            if (row >= n) continue;
#pragma unroll
            for (int ni = 0; ni < 2; ++ni) {
                const int col = c0 + 16 * (2 * wn + ni) + 4 * q;
                float h[4], dg[4], du[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, d;
                    ffn_act<decltype(ACT)::value, true>(acc[mi][ni][e], a, d);
                    const float up = acc[mi][ni + 2][e], g = dh[mi][ni][e];
                    h[e] = a * up;
                    dg[e] = g * up * d;
                    du[e] = g * a;
                }
                const int64_t left = f8 - col;
                store4(H + row * f8 + col, left, h);
                store4(dGU + row * 2 * f8 + col, left, dg);
                store4(dGU + row * 2 * f8 + f8 + col, left, du);
            }
        }
    });
}

// One product of k_ffn_dw: out (m x nn) = A^T B over the rows, A n x lda, B n x ldb.
template <typename T>
struct DwSide {
    const T* A;
    const T* B;
    int64_t lda, ldb;
    int m, nn;
    int tn, tiles;     // column tiles, all tiles (0: the product is not wanted)
    int64_t part;      // where its sums start in a chunk's partial sums
};

// Partial sums of both products over the rows of a chunk.
template <typename T, int MT, int NT>
__global__ void __launch_bounds__(kFfnThreads, 2)
k_ffn_dw(DwSide<T> p0, DwSide<T> p1, int64_t n, int64_t chunk, int64_t per_chunk, float* __restrict__ part) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ffn_lds<MT, NT>()];
    const int64_t u = xcd_unit(blockIdx.x, gridDim.x);
    const int tiles = p0.tiles + p1.tiles;
    const int64_t s = u / tiles;
    int t = (int)(u - s * tiles);
    const bool second = t >= p0.tiles;
    const DwSide<T> p = second ? p1 : p0;
    if (second) t -= p0.tiles;
    const int m0 = t / p.tn * (32 * MT), c0 = t % p.tn * (32 * NT);
    const int64_t r0 = s * chunk, rows = n - r0 < chunk ? n - r0 : chunk;
    floatx4 acc[MT][NT];
    zero_acc(acc);
    tile_product<T, false, false, MT, NT, false>({p.A + r0 * p.lda + m0, nullptr, p.lda, p.m - m0, rows},
                                                 {p.B + r0 * p.ldb + c0, nullptr, p.ldb, p.nn - c0, rows}, lds, acc);
    const int wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
    float* out = part + s * per_chunk + p.part;
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) {
        const int row = m0 + 16 * (MT * wm + mi) + i;
        if (row >= p.m) continue;
#pragma unroll
        for (int ni = 0; ni < NT; ++ni) {
            const int col = c0 + 16 * (NT * wn + ni) + 4 * q;
            const float v[4] = {acc[mi][ni][0], acc[mi][ni][1], acc[mi][ni][2], acc[mi][ni][3]};
            if (col < p.nn) store4(out + (int64_t)row * p.nn + col, p.nn - col, v);
        }
    }
}

// The weights' gradients from the chunks' sums, added in chunk order: per chunk dWg | dWu as ci x 2 f8, then dWd.
template <typename T>
__global__ void __launch_bounds__(kFfnThreads)
k_ffn_dw_sum(const float* __restrict__ part, int64_t chunks, int64_t per_chunk, int ci, int f, int f8, int co,
             T* __restrict__ dWg, T* __restrict__ dWu, T* __restrict__ dWd, int64_t up, int64_t total) {
    for (int64_t i = (int64_t)blockIdx.x * kFfnThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kFfnThreads) {
        T* out;
        if (i < up) {
            const int64_t row = i / (2 * f8);
            int col = (int)(i - row * 2 * f8);
            out = dWg;
            if (col >= f8) {
                out = dWu;
                col -= f8;
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

// A few rows (at most R): out (n x nn) = A B, or act(A B) * (A B2) with B2.  Bound: the weights, read once.  A
// thread takes 16 bytes of columns and every 64th reduction element; a block 4 x 16 bytes of
// columns, so that even a narrow layer is spread over many blocks.
constexpr int kFewCols = 4, kFewLanes = kFfnThreads / kFewCols;

template <typename T, int R, bool GATED>
__global__ void __launch_bounds__(kFfnThreads)
k_ffn_few(const T* __restrict__ A, int64_t lda, int n, int k, const T* __restrict__ B, const T* __restrict__ B2, int nn,
          int act, T* __restrict__ out, int64_t ldo) {
    typedef RowVec<T> RV;
    constexpr int V = RV::V, NB = GATED ? 2 : 1;
    __shared__ float red[kFfnThreads / 64][NB * R * V * kFewCols];
    const int cl = threadIdx.x % kFewCols, kl = threadIdx.x / kFewCols;
    const int col = (blockIdx.x * kFewCols + cl) * V;
    float acc[NB][R][V];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[b][r][e] = 0.f;
#pragma unroll 4
    for (int j = kl; j < k; j += kFewLanes) {
        typename RV::Raw w[NB];
        w[0] = load_vec<T, true>(B + (int64_t)j * nn + col, nn - col);
        if (GATED) w[NB - 1] = load_vec<T, true>(B2 + (int64_t)j * nn + col, nn - col);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float a = r < n ? to_f32(A[r * lda + j]) : 0.f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[b][r][e] = fmaf(a, RV::get(w[b], e), acc[b][r][e]);
        }
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float s = acc[b][r][e];
#pragma unroll
                for (int d = kFewCols; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
                if (lane < kFewCols) red[wave][((b * R + r) * kFewCols + cl) * V + e] = s;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < R * kFewCols * V; i += kFfnThreads) {
        const int r = i / (kFewCols * V), c = blockIdx.x * kFewCols * V + i % (kFewCols * V);
        float v[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v[b] = 0.f;
            for (int w = 0; w < kFfnThreads / 64; ++w) v[b] += red[w][b * R * kFewCols * V + i];
        }
        if (r >= n || c >= nn) continue;
        float o = v[0];
        if (GATED)
            with_act(act, [&](auto ACT) {
                float a, d;
                ffn_act<decltype(ACT)::value, false>(v[0], a, d);
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
static size_t ffn_size(int dtype) { return dtype == GSC_BF16 ? 2 : 4; }

// 16-row blocks a wave takes in a direction of `rows` outputs: 4 (tiles of 128) unless tiles of 64 leave
// less of the last one empty.
static bool ffn_narrow(int64_t rows) { return ceil_div(rows, 64) % 2 == 1 && rows < 512; }

static bool ffn_sizes_ok(int32_t dtype, int64_t n, int32_t ci, int32_t f, int32_t co) {
    return (dtype == GSC_F32 || dtype == GSC_BF16) && n >= 0 && ci >= 1 && f >= 1 && co >= 1 && ci <= kFfnMaxWidth &&
           f <= kFfnMaxWidth && co <= kFfnMaxWidth && n <= ((int64_t)1 << 31) * 16;
}

// Row tiles of 64 where 128 would leave compute units idle.
static bool ffn_short(int64_t n, int64_t col_tiles) { return ceil_div(n, 128) * col_tiles < 2 * device_cus(); }

template <typename T, bool BKC>
static void ffn_gemm(const T* A1, const T* A2, int64_t lda, int64_t n, int64_t ka, const T* B1, const T* B2, int64_t ldb,
                     int64_t kb, int co, T* Out, hipStream_t s) {
    const bool nar = ffn_narrow(co);
    const int nc = (int)ceil_div(co, nar ? 64 : 128);
    const bool sho = ffn_short(n, nc);
    auto* kern = sho ? (nar ? k_ffn_gemm<T, BKC, 2, 2> : k_ffn_gemm<T, BKC, 2, 4>)
                     : (nar ? k_ffn_gemm<T, BKC, 4, 2> : k_ffn_gemm<T, BKC, 4, 4>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(ceil_div(n, sho ? 64 : 128) * nc)), dim3(kFfnThreads), 0, s, A1, A2, lda,
                       n, ka, B1, B2, ldb, kb, co, Out, nc);
}

template <typename T>
static void ffn_fwd(const T* X, int64_t n, int ci, const T* Wg, const T* Wu, int f, const T* Wd, int co, int act, T* Y,
                    T* H, hipStream_t s) {
    const int64_t f8 = pad8(f);
    if (n <= kFfnFewRows) {
        constexpr int W = kFewCols * (16 / (int)sizeof(T));
        auto* up = n == 1 ? k_ffn_few<T, 1, true> : (n == 2 ? k_ffn_few<T, 2, true> : k_ffn_few<T, 4, true>);
        auto* down = n == 1 ? k_ffn_few<T, 1, false> : (n == 2 ? k_ffn_few<T, 2, false> : k_ffn_few<T, 4, false>);
        hipLaunchKernelGGL(up, dim3((unsigned)ceil_div(f, W)), dim3(kFfnThreads), 0, s, X, (int64_t)ci, (int)n, ci, Wg,
                           Wu, f, act, H, f8);
        hipLaunchKernelGGL(down, dim3((unsigned)ceil_div(co, W)), dim3(kFfnThreads), 0, s, H, f8, (int)n, f, Wd,
                           (const T*)nullptr, co, act, Y, (int64_t)co);
        return;
    }
    const int nf = (int)ceil_div(f, 64);
    const bool sho = ffn_short(n, nf);
    auto* up = sho ? k_ffn_up<T, 2> : k_ffn_up<T, 4>;
    hipLaunchKernelGGL(up, dim3((unsigned)(ceil_div(n, sho ? 64 : 128) * nf)), dim3(kFfnThreads), 0, s, X, n, ci, Wg, Wu, f, act, H, f8, nf);
    ffn_gemm<T, false>(H, nullptr, f8, n, f8, Wd, nullptr, co, f, co, Y, s);
}

// Row chunks of the weights' gradients: enough blocks for the device, at least 512 rows each.
constexpr int64_t kFfnChunkRows = 512;
static int64_t ffn_chunks(int64_t n, int64_t tiles) {
    int64_t c = ceil_div(4 * 256, tiles);
    const int64_t most = ceil_div(n, kFfnChunkRows);
    if (c > most) c = most;
    return c < 1 ? 1 : c;
}

struct FfnBwdLayout {
    int64_t f8, per_chunk, up, chunks, chunk;
    int m_nar, n_nar;   // tiles of 64 rows, of 64 columns
    int tn0, t0, tn1, t1;
    size_t h, dgu, part, total;
};

static FfnBwdLayout ffn_bwd_layout(int dtype, int64_t n, int ci, int f, int co) {
    FfnBwdLayout L;
    L.f8 = pad8(f);
    L.m_nar = ffn_narrow(ci);
    L.n_nar = ffn_narrow(co);
    const int bm = L.m_nar ? 64 : 128, bn = L.n_nar ? 64 : 128;
    L.tn0 = (int)ceil_div(2 * L.f8, bn);
    L.t0 = (int)ceil_div(ci, bm) * L.tn0;
    L.tn1 = (int)ceil_div(co, bn);
    L.t1 = (int)ceil_div(f, bm) * L.tn1;
    L.chunks = ffn_chunks(n, (int64_t)L.t0 + L.t1);
    L.chunk = ceil_div(ceil_div(n > 0 ? n : 1, L.chunks), 64) * 64;
    L.chunks = ceil_div(n > 0 ? n : 1, L.chunk);
    L.up = (int64_t)ci * 2 * L.f8;
    L.per_chunk = L.up + (int64_t)f * co;
    L.h = 0;
    L.dgu = ffn_al256((size_t)n * L.f8 * ffn_size(dtype));
    L.part = L.dgu + ffn_al256((size_t)n * 2 * L.f8 * ffn_size(dtype));
    L.total = L.part + ffn_al256((size_t)L.chunks * L.per_chunk * sizeof(float));
    return L;
}

template <typename T>
static void ffn_bwd(const FfnBwdLayout& L, const T* X, int64_t n, int ci, const T* Wg, const T* Wu, int f, const T* Wd,
                    int co, const T* dY, int act, T* dX, T* dWg, T* dWu, T* dWd, char* ws, hipStream_t s) {
    T* H = reinterpret_cast<T*>(ws + L.h);
    T* dGU = reinterpret_cast<T*>(ws + L.dgu);
    float* part = reinterpret_cast<float*>(ws + L.part);
    if (n > 0) {
        const int nf = (int)ceil_div(f, 64);
        const bool sho = ffn_short(n, nf);
        auto* mid = sho ? k_ffn_mid<T, 2> : k_ffn_mid<T, 4>;
        hipLaunchKernelGGL(mid, dim3((unsigned)(ceil_div(n, sho ? 64 : 128) * nf)), dim3(kFfnThreads), 0, s, X, dY, n, ci, co, Wg, Wu, Wd, f, act, H, dGU, (int)L.f8, nf);
        if (dX) ffn_gemm<T, true>(dGU, dGU + L.f8, 2 * L.f8, n, L.f8, Wg, Wu, f, f, ci, dX, s);
    }
    if (!dWg && !dWu && !dWd) return;
    const bool up = dWg || dWu;
    DwSide<T> p0{X, dGU, ci, 2 * L.f8, ci, (int)(2 * L.f8), L.tn0, up ? L.t0 : 0, 0};
    DwSide<T> p1{H, dY, L.f8, co, f, co, L.tn1, dWd ? L.t1 : 0, L.up};
    const int64_t chunks = n > 0 ? L.chunks : 0;
    if (n > 0) {
        auto* kern = L.m_nar ? (L.n_nar ? k_ffn_dw<T, 2, 2> : k_ffn_dw<T, 2, 4>)
                             : (L.n_nar ? k_ffn_dw<T, 4, 2> : k_ffn_dw<T, 4, 4>);
        hipLaunchKernelGGL(kern, dim3((unsigned)(chunks * (p0.tiles + p1.tiles))), dim3(kFfnThreads), 0, s, p0, p1, n,
                           L.chunk, L.per_chunk, part);
    }
    const int64_t total = dWd ? L.per_chunk : L.up;
    const int64_t blocks = ceil_div(total, kFfnThreads);
    hipLaunchKernelGGL(k_ffn_dw_sum<T>, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kFfnThreads), 0, s, part,
                       chunks, L.per_chunk, ci, f, (int)L.f8, co, dWg, dWu, dWd, L.up, total);
}

}  // namespace gsc

using namespace gsc;

extern "C" {

size_t gsc_gated_ffn_fwd_ws_bytes(int32_t dtype, int64_t n, int32_t c_in, int32_t hidden, int32_t c_out) {
    if (!ffn_sizes_ok(dtype, n, c_in, hidden, c_out)) return 0;
    return ffn_al256((size_t)n * pad8(hidden) * ffn_size(dtype));
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
    if (ceil_div(n, 64) * ceil_div(hidden > c_out ? hidden : c_out, 64) > 0x7fffffff)
        return fail(GSC_EINVAL, "gated_ffn_fwd: more tiles than a launch takes");
    if (n == 0) return GSC_OK;
    if (!X || !Wg || !Wu || !Wd || !Y) return fail(GSC_EINVAL, "gated_ffn_fwd: null X/Wg/Wu/Wd/Y");
    const size_t need = gsc_gated_ffn_fwd_ws_bytes(dtype, n, c_in, hidden, c_out);
    if (!ws || ws_bytes < need)
        return fail(GSC_ESHORT, "gated_ffn_fwd: ws needs %zu bytes, got %zu", need, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(GSC_EINVAL, "gated_ffn_fwd: ws must be aligned to 16 bytes");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == GSC_BF16)
        ffn_fwd<uint16_t>((const uint16_t*)X, n, c_in, (const uint16_t*)Wg, (const uint16_t*)Wu, hidden,
                          (const uint16_t*)Wd, c_out, act, (uint16_t*)Y, (uint16_t*)ws, s);
    else
        ffn_fwd<float>((const float*)X, n, c_in, (const float*)Wg, (const float*)Wu, hidden, (const float*)Wd, c_out,
                       act, (float*)Y, (float*)ws, s);
    GSC_LAUNCH_CHECK();
    return GSC_OK;
}

size_t gsc_gated_ffn_bwd_ws_bytes(int32_t dtype, int64_t n, int32_t c_in, int32_t hidden, int32_t c_out) {
    if (!ffn_sizes_ok(dtype, n, c_in, hidden, c_out)) return 0;
    return ffn_bwd_layout(dtype, n, c_in, hidden, c_out).total;
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
    const int widest = hidden > c_out ? (hidden > c_in ? hidden : c_in) : (c_out > c_in ? c_out : c_in);
    if (ceil_div(n, 64) * ceil_div(widest, 64) > 0x7fffffff)
        return fail(GSC_EINVAL, "gated_ffn_bwd: more tiles than a launch takes");
    if (!dX && !dWg && !dWu && !dWd) return GSC_OK;
    if (n == 0 && !dWg && !dWu && !dWd) return GSC_OK;
    if (n > 0 && (!X || !Wg || !Wu || !Wd || !dY)) return fail(GSC_EINVAL, "gated_ffn_bwd: null X/Wg/Wu/Wd/dY");
    const FfnBwdLayout L = ffn_bwd_layout(dtype, n, c_in, hidden, c_out);
    if (!ws || ws_bytes < L.total)
        return fail(GSC_ESHORT, "gated_ffn_bwd: ws needs %zu bytes, got %zu", L.total, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(GSC_EINVAL, "gated_ffn_bwd: ws must be aligned to 16 bytes");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == GSC_BF16)
        ffn_bwd<uint16_t>(L, (const uint16_t*)X, n, c_in, (const uint16_t*)Wg, (const uint16_t*)Wu, hidden,
                          (const uint16_t*)Wd, c_out, (const uint16_t*)dY, act, (uint16_t*)dX, (uint16_t*)dWg,
                          (uint16_t*)dWu, (uint16_t*)dWd, (char*)ws, s);
    else
        ffn_bwd<float>(L, (const float*)X, n, c_in, (const float*)Wg, (const float*)Wu, hidden, (const float*)Wd, c_out,
                       (const float*)dY, act, (float*)dX, (float*)dWg, (float*)dWu, (float*)dWd, (char*)ws, s);
    GSC_LAUNCH_CHECK();
    return GSC_OK;
}

}  // extern "C"
