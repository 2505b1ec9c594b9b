// Layer norm of feature rows, forward and backward.
//
//   m = mean(x),  v = mean((x - m)^2),  r = 1 / sqrt(v + eps),  h = (x - m) r,  y = h gamma + beta
//   g = dy gamma,  dx = r (g - mean(g) - h mean(g h)),  dgamma = sum over rows of dy h,  dbeta = sum of dy
//
// All sums are held in float32 (the sums over rows end in float64), in a fixed order: results are
// bit-reproducible.
//
// The mean is taken in two steps: m1 = x[0] + mean(x - x[0]) rounded to float32, then, with e = x - m1, its rest m2 =
// mean(e).  x - m is e - m2 and v is mean(e^2) - m2^2, both sums in one round of exchanges.  So neither an offset that a row's
// values share nor a first value far larger than the others costs digits.  (Nor does the difference: m2 is half a step of
// float32 at m1, which the deviation of a row that is not constant reaches, and the sum's roundings of x - x[0], a
// millionth of it, where the deviation is |x - x[0]| / sqrt(c) or more.)  The backward pass gets m1 + m2 rounded to float32,
// and where a row's values share an offset that rounding is as large as their deviations: it takes x - mean, and out of that
// the rest's mean, again.
//
// Bound: HBM (a read and a write of n x c forward, two reads and a write backward).  A row stays
// in the registers of LPR lanes (NV pieces of 16 bytes a lane), so it is read once; a wave holds
// 64 / LPR rows, reduces each with log2(LPR) lane exchanges and needs no LDS, and the lanes keep
// their columns' gamma, beta and (backward) column sums in registers over all rows they visit.
// Measured: 300,000 rows of 256 bfloat16 columns forward 56 us (5.5 TB/s), backward 91 us and 4 us for the sums (5.0 TB/s);
// 20,011 rows of 1,027 (rows at odd addresses, a third of the lanes idle in the last piece) 21 and 36 us (3.8 and 3.5 TB/s);
// 20,000 rows of 4,096 bfloat16 columns, element by element, forward 212 us, backward 236 us (1.5 and 2.1 TB/s).
// Rows of more than kLnRegCols columns take a block each and are read again for each sum (from the L2); with the sums over
// rows the backward pass is a block a row for the rows' means, and then a thread a column for dX and the sums.
#include "row_vec.h"

namespace gsc {

constexpr int kLnThreads = 256;
constexpr int kLnRegCols = 2048;       // 32 elements a lane of a wave
constexpr int kLnMaxCols = 1 << 30;
constexpr int64_t kLnFwdBlocks = 2048;  // blocks that walk over the rows (8 a CU)
constexpr int64_t kLnChunks = 1024;     // row chunks (blocks) of the backward pass: as many partial column sums
// Wide rows with many elements a lane take half as many of either: fewer blocks fit a CU, and the columns' arrays and sums that
// a block starts and ends with are long (bfloat16 backward, 20,000 rows of 1,024 columns 28 us, 30 with all of them; 205,400
// rows of 100 columns 44 and 31; float32, 79,922 rows of 257 columns in 12 elements a lane 53 and 45).
static int64_t ln_most(int c, int per_lane, int64_t most) { return c > 256 && per_lane >= 16 ? most / 2 : most; }
constexpr int kLnSumCh = 16, kLnSumLanes = 64;
constexpr int64_t kLnSumBlocks = 65536;   // (a launch takes fewer than 2^32 threads: 2^22 blocks of these)

static int64_t ln_row_blocks(int64_t n, int rows, int64_t most) {
    const int64_t b = (n + rows - 1) / rows;
    return b < 1 ? 1 : (b > most ? most : b);
}

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int d = LPR / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// V values of a per-column float32 array (null: the value `none`), 0 behind its end: 16-byte loads, which a wave
// pays for once over all of its rows (element by element they took longer than a row did).
template <int V>
__device__ __forceinline__ void load_cols(const float* p, int col, int c, float none, float (&v)[V]) {
#pragma unroll
    for (int h = 0; h < V; h += 4) {
        RowVec<float>::Raw r = {0, 0, 0, 0};
        if (p) r = load_vec<float, true>(p + col + h, c - col - h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[h + e] = p ? __uint_as_float(r[e]) : (col + h + e < c ? none : 0.f);
    }
}

// Whether piece i of every lane is a whole one (the shapes of ln_dispatch but the widest need all their pieces).
template <int NV>
constexpr bool ln_whole(int i) { return i < NV - 1 && NV <= 4; }

// A row's pieces of one lane: piece i holds the V elements from column (i LPR + l) V on, zeros behind the end.  A partial
// piece is the row's last 16 bytes, shifted (loads of its elements one by one took as long as the rest of the row).
template <typename T, int LPR, int NV, bool TAIL>
__device__ __forceinline__ void load_row(const T* x, int l, int c, typename RowVec<T>::Raw (&raw)[NV]) {
    constexpr int V = RowVec<T>::V;
    typedef typename RowVec<T>::Raw Raw;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * LPR + l) * V;
        if (ln_whole<NV>(i)) raw[i] = *reinterpret_cast<const Raw*>(x + col);
        else if (!TAIL || c < V) raw[i] = load_vec<T, TAIL>(x + col, c - col);
        else raw[i] = load_last<T>(x, col, c);
    }
}
// ... and back: the partial piece in stores of 8, 4 and 2 bytes.
template <typename T, int NV, bool TAIL>
__device__ __forceinline__ void store_piece(T* y, int i, int col, int c, const float (&v)[RowVec<T>::V]) {
    typedef RowVec<T> R;
    typedef typename R::Raw Raw;
    if (ln_whole<NV>(i) || col + R::V <= c) {
        *reinterpret_cast<Raw*>(y + col) = R::put(v);
    } else if (TAIL && col < c) {
        const Raw r = R::put(v);
        uint32_t* p = reinterpret_cast<uint32_t*>(y + col);   // (at any element's address)
        const int bytes = (c % R::V) * (int)sizeof(T);
        if (bytes & 8) {
            typedef uint32_t Two __attribute__((ext_vector_type(2), aligned(2)));
            *reinterpret_cast<Two*>(p) = Two{r[0], r[1]};
        }
        if (bytes & 4) {
            typedef uint32_t One __attribute__((aligned(2)));
            *reinterpret_cast<One*>(p + (bytes >> 3) * 2) = bytes & 8 ? r[2] : r[0];
        }
        if (sizeof(T) == 2 && (bytes & 2)) {
            const uint32_t w = bytes & 8 ? (bytes & 4 ? r[3] : r[2]) : (bytes & 4 ? r[1] : r[0]);
            *reinterpret_cast<uint16_t*>(p + (bytes >> 2)) = (uint16_t)w;
        }
    }
}

template <typename T, int LPR, int NV, bool TAIL>
__global__ void __launch_bounds__(kLnThreads) k_ln_fwd(const T* X, int64_t n, int c, const float* __restrict__ gamma,
                                                       const float* __restrict__ beta, float eps, T* Y,
                                                       float* __restrict__ mean, float* __restrict__ rstd) {
    typedef RowVec<T> R;
    constexpr int V = R::V, RPB = kLnThreads / LPR;
    const int l = threadIdx.x % LPR;
    const float inv_c = 1.f / (float)c;
    float ga[NV][V], be[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_cols<V>(gamma, (i * LPR + l) * V, c, 1.f, ga[i]);
        load_cols<V>(beta, (i * LPR + l) * V, c, 0.f, be[i]);
    }
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR; row < n; row += (int64_t)gridDim.x * RPB) {
        typename R::Raw raw[NV];
        load_row<T, LPR, NV, TAIL>(X + row * c, l, c, raw);
        const float x0 = __shfl(R::get(raw[0], 0), 0, LPR);   // the row's first element
        float v[NV][V], s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool in = ln_whole<NV>(i) || (i * LPR + l) * V + (TAIL ? e : 0) < c;
                s += in ? R::get(raw[i], e) - x0 : 0.f;
            }
        const float m1 = x0 + row_sum<LPR>(s) * inv_c;
        float t = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool in = ln_whole<NV>(i) || (i * LPR + l) * V + (TAIL ? e : 0) < c;
                v[i][e] = in ? R::get(raw[i], e) - m1 : 0.f;
                t += v[i][e];
                q = fmaf(v[i][e], v[i][e], q);
            }
        const float m2 = row_sum<LPR>(t) * inv_c;
        const float r = 1.f / sqrtf(fmaf(-m2, m2, row_sum<LPR>(q) * inv_c) + eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * LPR + l) * V;
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = fmaf((v[i][e] - m2) * r, ga[i][e], be[i][e]);
            store_piece<T, NV, TAIL>(Y + row * c, i, col, c, o);
        }
        if (l == 0) {
            if (mean) mean[row] = m1 + m2;
            if (rstd) rstd[row] = r;
        }
    }
}

// Sum over a block's threads (every thread gets it); sh: one float per wave.
__device__ __forceinline__ float ln_block_sum(float v, float* sh) {
    v = row_sum<64>(v);
    __syncthreads();   // the previous sum is read
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < kLnThreads / 64; ++w) v += sh[w];
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kLnThreads) k_ln_fwd_wide(const T* X, int64_t n, int c,
                                                            const float* __restrict__ gamma,
                                                            const float* __restrict__ beta, float eps, T* Y,
                                                            float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float sh[kLnThreads / 64];
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* x = X + row * c;
        const float x0 = to_f32(x[0]);
        float s = 0.f, t = 0.f, q = 0.f;
        for (int i = threadIdx.x; i < c; i += kLnThreads) s += to_f32(x[i]) - x0;
        const float m1 = x0 + ln_block_sum(s, sh) / (float)c;
        for (int i = threadIdx.x; i < c; i += kLnThreads) {
            const float e = to_f32(x[i]) - m1;
            t += e;
            q = fmaf(e, e, q);
        }
        const float m2 = ln_block_sum(t, sh) / (float)c;
        const float r = 1.f / sqrtf(fmaf(-m2, m2, ln_block_sum(q, sh) / (float)c) + eps);   // (every thread has read x[0])
        for (int i = threadIdx.x; i < c; i += kLnThreads)
            store_out(&Y[row * c + i],
                      fmaf((to_f32(x[i]) - m1 - m2) * r, gamma ? gamma[i] : 1.f, beta ? beta[i] : 0.f));
        if (threadIdx.x == 0) {
            if (mean) mean[row] = m1 + m2;
            if (rstd) rstd[row] = r;
        }
    }
}

// An element of dX (the same operations wherever it is formed), a = mean(g), b = mean(g h).
__device__ __forceinline__ float ln_dx(float dy, float ga, float h, float r, float a, float b) {
    return r * fmaf(-h, b, fmaf(dy, ga, -a));
}

// part: per block, the c column sums of dy h, then of dy.
template <typename T, int LPR, int NV, bool TAIL>
__global__ void __launch_bounds__(kLnThreads) k_ln_bwd(const T* X, const T* dY, int64_t n, int c,
                                                       const float* __restrict__ gamma,
                                                       const float* __restrict__ mean, const float* __restrict__ rstd,
                                                       T* dX, float* __restrict__ part) {
    typedef RowVec<T> R;
    constexpr int V = R::V, RPB = kLnThreads / LPR;
    extern __shared__ float ln_red[];   // waves x c
    const int l = threadIdx.x % LPR;
    const float inv_c = 1.f / (float)c;
    float ga[NV][V], sg[NV][V], sb[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_cols<V>(gamma, (i * LPR + l) * V, c, 1.f, ga[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) sg[i][e] = sb[i][e] = 0.f;
    }
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR; row < n; row += (int64_t)gridDim.x * RPB) {
        typename R::Raw xr[NV], yr[NV];
        load_row<T, LPR, NV, TAIL>(X + row * c, l, c, xr);
        load_row<T, LPR, NV, TAIL>(dY + row * c, l, c, yr);
        const float m = mean[row], r = rstd[row];
        float t = 0.f, a = 0.f, b = 0.f;   // sums of x - m, of g and of g (x - m)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool in = ln_whole<NV>(i) || (i * LPR + l) * V + (TAIL ? e : 0) < c;
                const float d = in ? R::get(xr[i], e) - m : 0.f;
                const float g = R::get(yr[i], e) * ga[i][e];
                t += d;
                a += g;
                b = fmaf(g, d, b);
            }
        const float m2 = row_sum<LPR>(t) * inv_c;
        a = row_sum<LPR>(a) * inv_c;
        b = fmaf(-m2, a, row_sum<LPR>(b) * inv_c) * r;   // mean of g h
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * LPR + l) * V;
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = (R::get(xr[i], e) - m - m2) * r, d = R::get(yr[i], e);
                sg[i][e] = fmaf(d, h, sg[i][e]);   // (behind the row's end dy is 0, and no column is stored)
                sb[i][e] += d;
                o[e] = ln_dx(d, ga[i][e], h, r, a, b);
            }
            if (dX) store_piece<T, NV, TAIL>(dX + row * c, i, col, c, o);
        }
    }
    if (!part) return;
    // the rows of a wave, then the waves, in a fixed order
    const int w = threadIdx.x >> 6;
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float s = k ? sb[i][e] : sg[i][e];
#pragma unroll
                for (int d = LPR; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
                const int col = (i * LPR + l) * V + e;
                if ((threadIdx.x & 63) < LPR && col < c) ln_red[w * c + col] = s;
            }
        __syncthreads();
        for (int col = threadIdx.x; col < c; col += kLnThreads) {
            float s = 0.f;
            for (int u = 0; u < kLnThreads / 64; ++u) s += ln_red[u * c + col];
            part[((int64_t)blockIdx.x * 2 + k) * c + col] = s;
        }
        __syncthreads();
    }
}

// dX, or, with `rows`, what it (or, where it is null, what the sums over rows) takes of each row: m2, mean(g) and mean(g h).
template <typename T>
__global__ void __launch_bounds__(kLnThreads) k_ln_bwd_wide(const T* X, const T* dY, int64_t n, int c,
                                                            const float* __restrict__ gamma,
                                                            const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, T* dX,
                                                            float* __restrict__ rows) {
    __shared__ float sh[kLnThreads / 64];
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* x = X + row * c;
        const T* dy = dY + row * c;
        const float m = mean[row], r = rstd[row];
        float t = 0.f, a = 0.f, b = 0.f;
        if (!dX) {
            for (int i = threadIdx.x; i < c; i += kLnThreads) t += to_f32(x[i]) - m;
            t = ln_block_sum(t, sh) / (float)c;
            if (threadIdx.x == 0) rows[3 * row] = t;
            continue;
        }
        for (int i = threadIdx.x; i < c; i += kLnThreads) {
            const float g = to_f32(dy[i]) * (gamma ? gamma[i] : 1.f), d = to_f32(x[i]) - m;
            t += d;
            a += g;
            b = fmaf(g, d, b);
        }
        const float m2 = ln_block_sum(t, sh) / (float)c;
        a = ln_block_sum(a, sh) / (float)c;
        b = fmaf(-m2, a, ln_block_sum(b, sh) / (float)c) * r;
        if (rows) {
            if (threadIdx.x == 0) rows[3 * row] = m2, rows[3 * row + 1] = a, rows[3 * row + 2] = b;
            continue;
        }
        for (int i = threadIdx.x; i < c; i += kLnThreads) {
            const float h = (to_f32(x[i]) - m - m2) * r;
            store_out(&dX[row * c + i], ln_dx(to_f32(dy[i]), gamma ? gamma[i] : 1.f, h, r, a, b));
        }
    }
}

// Column sums of wide rows and, unless null, dX: a thread takes a column of a chunk's rows.
template <typename T>
__global__ void __launch_bounds__(kLnThreads) k_ln_bwd_wide_cols(const T* X, const T* dY, int64_t n, int c,
                                                                 const float* __restrict__ gamma,
                                                                 const float* __restrict__ mean,
                                                                 const float* __restrict__ rstd,
                                                                 const float* __restrict__ rows, T* dX,
                                                                 float* __restrict__ part) {
    const int64_t chunks = gridDim.x, k = blockIdx.x;
    const int64_t r0 = n * k / chunks, r1 = n * (k + 1) / chunks;
    for (int col = blockIdx.y * kLnThreads + threadIdx.x; col < c; col += gridDim.y * kLnThreads) {
        float sg = 0.f, sb = 0.f;
        const float ga = gamma ? gamma[col] : 1.f;
        auto add = [&](int64_t row, T x, T dy) {
            const float r = rstd[row], d = to_f32(dy), h = (to_f32(x) - mean[row] - rows[3 * row]) * r;
            sg = fmaf(d, h, sg);
            sb += d;
            if (dX) store_out(&dX[row * c + col], ln_dx(d, ga, h, r, rows[3 * row + 1], rows[3 * row + 2]));
        };
        int64_t row = r0;
        for (; row + 4 <= r1; row += 4) {   // (four rows are read before the first is written: dX may be X or dY)
            T x[4], dy[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = X[(row + i) * c + col], dy[i] = dY[(row + i) * c + col];
#pragma unroll
            for (int i = 0; i < 4; ++i) add(row + i, x[i], dy[i]);
        }
        for (; row < r1; ++row) add(row, X[row * c + col], dY[row * c + col]);
        part[k * 2 * c + col] = sg;
        part[(k * 2 + 1) * c + col] = sb;
    }
}

// The 2 c column sums from the chunks' sums: lane l of a column adds chunks l, l + 64, ... in
// float64, then the lanes' sums pairwise.
__global__ void __launch_bounds__(kLnSumCh * kLnSumLanes)
k_ln_bwd_sum(const float* __restrict__ part, int64_t chunks, int c, float* __restrict__ dgamma,
             float* __restrict__ dbeta) {
    __shared__ double sh[kLnSumLanes][kLnSumCh];
    const int ci = threadIdx.x % kLnSumCh, l = threadIdx.x / kLnSumCh;
    const int64_t c2 = 2 * (int64_t)c;
    for (int64_t ch0 = (int64_t)blockIdx.x * kLnSumCh; ch0 < c2; ch0 += (int64_t)gridDim.x * kLnSumCh) {
        const int64_t ch = ch0 + ci;
        double a = 0.0;
        if (ch < c2) {
#pragma unroll 4
            for (int64_t k = l; k < chunks; k += kLnSumLanes) a += part[k * c2 + ch];
        }
        __syncthreads();   // the previous columns' sums are read
        sh[l][ci] = a;
        for (int d = kLnSumLanes / 2; d > 0; d >>= 1) {
            __syncthreads();
            if (l < d) sh[l][ci] += sh[l + d][ci];
        }
        if (l == 0 && ch < c2) {
            if (ch < c) {
                if (dgamma) dgamma[ch] = (float)sh[0][ci];
            } else if (dbeta) {
                dbeta[ch - c] = (float)sh[0][ci];
            }
        }
    }
}

// f(LPR, NV, TAIL as constants) for rows of c <= kLnRegCols columns: of the shapes of at most MOST pieces a lane the one
// that holds the row with the fewest pieces in all, with more lanes a row among equals; a whole wave
// with more pieces for the widest rows.
template <typename T, int MOST, typename F>
static void ln_dispatch(int c, F f) {
    constexpr int V = RowVec<T>::V;
    const int vecs = (c + V - 1) / V;
    const bool tail = c % V != 0;
    int lpr = 64, nv = (vecs + 63) / 64;
    for (int l = 32; l >= 8; l /= 2) {
        const int k = (vecs + l - 1) / l;
        if (k <= MOST && l * k < lpr * nv) lpr = l, nv = k;
    }
    auto with = [&](auto LPR, auto NV) {
        if (tail) f(LPR, NV, std::true_type{});
        else f(LPR, NV, std::false_type{});
    };
    auto pieces = [&](auto LPR) {
        if (nv == 1) return with(LPR, std::integral_constant<int, 1>{});
        if (nv == 2) return with(LPR, std::integral_constant<int, 2>{});
        if (nv == 3) return with(LPR, std::integral_constant<int, 3>{});
        if constexpr (MOST > 3 || decltype(LPR)::value == 64)
            if (nv == 4) return with(LPR, std::integral_constant<int, 4>{});
        if constexpr (V == 4 && decltype(LPR)::value == 64) {   // float32 rows: up to 512 pieces
            if (nv <= 6) return with(LPR, std::integral_constant<int, 6>{});
            return with(LPR, std::integral_constant<int, 8>{});
        }
    };
    if (lpr == 64) pieces(std::integral_constant<int, 64>{});
    else if (lpr == 32) pieces(std::integral_constant<int, 32>{});
    else if (lpr == 16) pieces(std::integral_constant<int, 16>{});
    else pieces(std::integral_constant<int, 8>{});
}

template <typename T>
static void ln_fwd(const void* X_, int64_t n, int c, const float* gamma, const float* beta, float eps, void* Y_,
                   float* mean, float* rstd, hipStream_t s) {
    const T* X = reinterpret_cast<const T*>(X_);
    T* Y = reinterpret_cast<T*>(Y_);
    if (c > kLnRegCols) {
        hipLaunchKernelGGL(k_ln_fwd_wide<T>, dim3((unsigned)ln_row_blocks(n, 1, kLnFwdBlocks)), dim3(kLnThreads), 0, s,
                           X, n, c, gamma, beta, eps, Y, mean, rstd);
        return;
    }
    ln_dispatch<T, 3>(c, [&](auto LPR, auto NV, auto TAIL) {
        constexpr int L = decltype(LPR)::value, N = decltype(NV)::value;
        auto* kern = k_ln_fwd<T, L, N, decltype(TAIL)::value>;
        const int64_t blocks = ln_row_blocks(n, kLnThreads / L, ln_most(c, N * RowVec<T>::V, kLnFwdBlocks));
        hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kLnThreads), 0, s, X, n, c, gamma, beta, eps, Y, mean, rstd);
    });
}

// Floats of the workspace: the chunks' column sums, then (wide rows) three of each row.
static size_t ln_part(int64_t n, int c) { return (size_t)ln_row_blocks(n, kLnThreads / 64, kLnChunks) * 2 * (size_t)c; }

// Launches the passes over the rows; returns the number of chunks whose sums are in part.
template <typename T>
static int64_t ln_bwd(const void* X_, const void* dY_, int64_t n, int c, const float* gamma, const float* mean,
                      const float* rstd, void* dX_, float* part, hipStream_t s) {
    const T* X = reinterpret_cast<const T*>(X_);
    const T* dY = reinterpret_cast<const T*>(dY_);
    T* dX = reinterpret_cast<T*>(dX_);
    int64_t chunks = 0;
    if (c > kLnRegCols) {
        // of 64 rows, or of fewer, down to 8, while there are under 1,024 blocks (300 rows of 8,192 bfloat16 columns: 23 us,
        // 29)
        const unsigned cb = (unsigned)((c + kLnThreads - 1) / kLnThreads);
        const int64_t most = ln_row_blocks(n, 8, 1024 / cb + 1);
        chunks = ln_row_blocks(n, 64, kLnChunks);
        if (chunks < most) chunks = most;
        float* rows = part ? part + ln_part(n, c) : nullptr;
        if (n > 0)
            hipLaunchKernelGGL(k_ln_bwd_wide<T>, dim3((unsigned)ln_row_blocks(n, 1, kLnFwdBlocks)), dim3(kLnThreads),
                               0, s, X, dY, n, c, gamma, mean, rstd, dX, rows);
        if (part)
            hipLaunchKernelGGL(k_ln_bwd_wide_cols<T>, dim3((unsigned)chunks, cb < 4096 ? cb : 4096), dim3(kLnThreads),
                               0, s, X, dY, n, c, gamma, mean, rstd, rows, dX, part);
        return chunks;
    }
    ln_dispatch<T, 3>(c, [&](auto LPR, auto NV, auto TAIL) {
        constexpr int L = decltype(LPR)::value, N = decltype(NV)::value;
        auto* kern = k_ln_bwd<T, L, N, decltype(TAIL)::value>;
        chunks = ln_row_blocks(n, kLnThreads / L, ln_most(c, N * RowVec<T>::V, kLnChunks));
        hipLaunchKernelGGL(kern, dim3((unsigned)chunks), dim3(kLnThreads),
                           part ? (kLnThreads / 64) * c * sizeof(float) : 0, s, X, dY, n, c, gamma, mean, rstd, dX,
                           part);
    });
    return chunks;
}

}  // namespace gsc

using namespace gsc;

extern "C" {

int gsc_layer_norm_fwd(int32_t dtype, const void* X, int64_t n, int32_t c, const float* gamma, const float* beta,
                       float eps, void* Y, float* mean, float* rstd, void* stream) {
    clear_error();
    if (dtype != GSC_F32 && dtype != GSC_BF16) return fail(GSC_EINVAL, "layer_norm_fwd: unknown dtype %d", dtype);
    if (n < 0 || c < 1 || c > kLnMaxCols) return fail(GSC_EINVAL, "layer_norm_fwd: bad sizes n=%lld c=%d", (long long)n, c);
    if (!(eps >= 0.f) || eps > 3.4e38f) return fail(GSC_EINVAL, "layer_norm_fwd: eps must be finite and not negative");
    if (n == 0) return GSC_OK;
    if (!X || !Y) return fail(GSC_EINVAL, "layer_norm_fwd: null X/Y");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == GSC_BF16) ln_fwd<uint16_t>(X, n, c, gamma, beta, eps, Y, mean, rstd, s);
    else ln_fwd<float>(X, n, c, gamma, beta, eps, Y, mean, rstd, s);
    GSC_LAUNCH_CHECK();
    return GSC_OK;
}

size_t gsc_layer_norm_bwd_ws_bytes(int64_t n, int32_t c) {
    if (n < 0 || c < 1 || c > kLnMaxCols) return 0;
    return (ln_part(n, c) + (c > kLnRegCols ? 3 * (size_t)n : 0)) * sizeof(float);
}

int gsc_layer_norm_bwd(int32_t dtype, const void* X, const void* dY, int64_t n, int32_t c, const float* gamma,
                       const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta, void* ws,
                       size_t ws_bytes, void* stream) {
    clear_error();
    if (dtype != GSC_F32 && dtype != GSC_BF16) return fail(GSC_EINVAL, "layer_norm_bwd: unknown dtype %d", dtype);
    if (n < 0 || c < 1 || c > kLnMaxCols) return fail(GSC_EINVAL, "layer_norm_bwd: bad sizes n=%lld c=%d", (long long)n, c);
    if (n > 0 && (!X || !dY || !mean || !rstd)) return fail(GSC_EINVAL, "layer_norm_bwd: null X/dY/mean/rstd");
    const bool sums = dgamma || dbeta;
    if (sums) {
        const size_t need = gsc_layer_norm_bwd_ws_bytes(n, c);
        if (!ws || ws_bytes < need)
            return fail(GSC_ESHORT, "layer_norm_bwd: ws needs %zu bytes, got %zu", need, ws ? ws_bytes : (size_t)0);
        if (reinterpret_cast<uintptr_t>(ws) % alignof(float))
            return fail(GSC_EINVAL, "layer_norm_bwd: ws must be aligned to 4 bytes");
    }
    if (!sums && (!dX || n == 0)) return GSC_OK;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    float* part = sums ? reinterpret_cast<float*>(ws) : nullptr;
    const int64_t chunks = dtype == GSC_BF16 ? ln_bwd<uint16_t>(X, dY, n, c, gamma, mean, rstd, dX, part, s)
                                             : ln_bwd<float>(X, dY, n, c, gamma, mean, rstd, dX, part, s);
    GSC_LAUNCH_CHECK();
    if (sums) {
        hipLaunchKernelGGL(k_ln_bwd_sum, dim3((unsigned)ln_row_blocks(2 * (int64_t)c, kLnSumCh, kLnSumBlocks)),
                           dim3(kLnSumCh * kLnSumLanes), 0, s, part, chunks, c, dgamma, dbeta);
        GSC_LAUNCH_CHECK();
    }
    return GSC_OK;
}

}  // extern "C"
