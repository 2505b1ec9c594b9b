// Rotary positions with several axes: pairs of a head's channels turned by angles that follow the
// row's coordinates.  Pair j of axis a (P_a pairs) turns by
//
//   t = x_a scale_a base^(-j / P_a),   (u, v) -> (u cos t - v sin t, u sin t + v cos t),
//
// and by -t with `inverse` (the gradient of the rotation, and its undoing).
//
// The angle is worked out in float64 as a number of turns and brought into half a turn either way
// before it is rounded (a coordinate of 10^6 leaves no digits of a float32 angle); sine and cosine
// follow in float32, the rotation in float32, rounded once as it is stored.
//
// Bound: HBM (a read and a write of the heads).  An angle serves all heads of a row, so a block takes
// kRotRows rows at most, puts the cosines and sines of their pairs into LDS, one evaluation per
// row and pair, and then streams the rows' heads past them in pieces of 16 bytes.  The frequencies
// (one float64 power per pair) are worked out once per block; blocks walk over the rows.  300,000 rows of 16 heads of 32
// bfloat16 channels in rows of 768: 132 us (4.7 TB/s); 120,011 rows of 6 heads of 64 float32 channels 73 us (5.1 TB/s).
#include "row_vec.h"

namespace gsc {

constexpr int kRotThreads = 256;
constexpr int kRotRows = 64;            // rows of a block's step at most
constexpr int kRotLds = 32768;          // bytes of cosines and sines at most
constexpr int kRotMaxHead = 4096;       // channels of a head
constexpr int kRotMaxAxes = 7;
constexpr int64_t kRotBlocks = 2048;

struct RotAxes {
    int end[kRotMaxAxes];        // axis a has pairs [end[a - 1], end[a])
    double scale[kRotMaxAxes];   // in turns: scale_a / (2 pi)
    double log2_base;
    int D;
};

// ADJ: pair p is channels (2 p, 2 p + 1) of a head, else (p, p + d / 2).  A thread takes a group of VP
// consecutive pairs of a head: 16 bytes (ADJ), or 16 bytes of either half.
template <typename T, bool ADJ, bool TAIL>
__global__ void __launch_bounds__(kRotThreads) k_rotary(const T* X, int64_t n, int heads, int d, int64_t ldx,
                                                        const int32_t* __restrict__ coords, RotAxes ax, int rows,
                                                        float sign, T* Y, int64_t ldy) {
    typedef RowVec<T> R;
    constexpr int V = R::V, VP = ADJ ? V / 2 : V;
    extern __shared__ __attribute__((aligned(16))) double rot_lds[];
    const int np = ax.end[ax.D - 1];            // pairs that turn
    double* freq = rot_lds;                      // turns per unit of the coordinate, np
    float2* cs = reinterpret_cast<float2*>(rot_lds + np);   // cosine and sine: rows x np
    auto axis_of = [&](int p) {
        int a = 0;
#pragma unroll
        for (int i = 0; i < kRotMaxAxes - 1; ++i)
            if (i < ax.D - 1 && p >= ax.end[i]) a = i + 1;
        return a;
    };
    auto pick = [&](int a, auto get) {   // get(a) with constant indices of the argument's arrays
        auto v = get(0);
#pragma unroll
        for (int i = 1; i < kRotMaxAxes; ++i)
            if (a == i) v = get(i);
        return v;
    };
    for (int p = threadIdx.x; p < np; p += kRotThreads) {
        const int a = axis_of(p);
        const int first = a ? pick(a - 1, [&](int i) { return ax.end[i]; }) : 0;
        const int cnt = pick(a, [&](int i) { return ax.end[i]; }) - first;
        freq[p] = pick(a, [&](int i) { return ax.scale[i]; }) * exp2(-(double)(p - first) / (double)cnt * ax.log2_base);
    }
    const int half = d >> 1;
    const int groups = (half + VP - 1) / VP, per_row = heads * groups;
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < n; r0 += (int64_t)gridDim.x * rows) {
        const int nr = (int)(n - r0 < rows ? n - r0 : rows);
        __syncthreads();   // the frequencies are there; the previous rows' angles are read
        for (int i = threadIdx.x; i < nr * np; i += kRotThreads) {
            const int r = i / np, p = i - r * np;
            const double t = (double)coords[(r0 + r) * (1 + ax.D) + 1 + axis_of(p)] * freq[p];
            float sn, cn;
            sincospif((float)(2.0 * (t - rint(t))), &sn, &cn);
            cs[i] = make_float2(cn, sign * sn);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < nr * per_row; i += kRotThreads) {
            const int r = i / per_row, k = i - r * per_row;
            const int h = k / groups, p0 = (k - h * groups) * VP;
            const float2* w = cs + r * np;
            const T* x = X + (r0 + r) * ldx + (int64_t)h * d;
            T* y = Y + (r0 + r) * ldy + (int64_t)h * d;
            if (ADJ) {
                const int left = d - 2 * p0;
                const typename R::Raw a = load_vec<T, TAIL>(x + 2 * p0, left);
                float o[V];
#pragma unroll
                for (int e = 0; e < VP; ++e) {
                    const float u = R::get(a, 2 * e), v = R::get(a, 2 * e + 1);
                    o[2 * e] = u;
                    o[2 * e + 1] = v;
                    if (p0 + e < np) {
                        const float2 q = w[p0 + e];
                        o[2 * e] = u * q.x - v * q.y;
                        o[2 * e + 1] = u * q.y + v * q.x;
                    }
                }
                store_vec<T, TAIL>(y + 2 * p0, left, o);
            } else {
                const int left = half - p0;
                const typename R::Raw a = load_vec<T, TAIL>(x + p0, left), b = load_vec<T, TAIL>(x + half + p0, left);
                float o0[V], o1[V];
#pragma unroll
                for (int e = 0; e < VP; ++e) {
                    const float u = R::get(a, e), v = R::get(b, e);
                    o0[e] = u;
                    o1[e] = v;
                    if (p0 + e < np) {
                        const float2 q = w[p0 + e];
                        o0[e] = u * q.x - v * q.y;
                        o1[e] = u * q.y + v * q.x;
                    }
                }
                store_vec<T, TAIL>(y + p0, left, o0);
                store_vec<T, TAIL>(y + half + p0, left, o1);
            }
        }
    }
}

template <typename T>
static void rotary(const void* X, int64_t n, int heads, int d, int64_t ldx, const int32_t* coords, const RotAxes& ax,
                   bool adj, float sign, void* Y, int64_t ldy, hipStream_t s) {
    constexpr int V = RowVec<T>::V;
    const int np = ax.end[ax.D - 1];
    const int vp = adj ? V / 2 : V, half = d / 2;
    const bool tail = half % vp != 0;
    const int64_t per_row = (int64_t)heads * ((half + vp - 1) / vp);
    // about four pieces a thread, fewer rows where there are not enough of them for the device
    int64_t rows = (4 * kRotThreads + per_row - 1) / per_row;
    const int64_t spread = (n + 2 * device_cus() - 1) / (2 * device_cus());
    if (rows > spread) rows = spread;
    if (rows > kRotRows) rows = kRotRows;
    if (np > 0 && rows > kRotLds / (8 * np)) rows = kRotLds / (8 * np);
    if (rows < 1) rows = 1;
    const int64_t steps = (n + rows - 1) / rows;
    auto* kern = adj ? (tail ? k_rotary<T, true, true> : k_rotary<T, true, false>)
                     : (tail ? k_rotary<T, false, true> : k_rotary<T, false, false>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(steps < kRotBlocks ? steps : kRotBlocks)), dim3(kRotThreads),
                       (size_t)(8 * np + 8 * np * rows), s, reinterpret_cast<const T*>(X), n, heads, d, ldx, coords, ax,
                       (int)rows, sign, reinterpret_cast<T*>(Y), ldy);
}

}  // namespace gsc

using namespace gsc;

extern "C" {

int gsc_rotary(int32_t dtype, const void* X, int64_t n, int32_t heads, int32_t d, int64_t ldx, const int32_t* coords,
               int32_t D, const int32_t* axis_pairs, const double* axis_scale, double base, int32_t pairing,
               int32_t inverse, void* Y, int64_t ldy, void* stream) {
    clear_error();
    if (dtype != GSC_F32 && dtype != GSC_BF16) return fail(GSC_EINVAL, "rotary: unknown dtype %d", dtype);
    if (pairing != GSC_ROTARY_ADJACENT && pairing != GSC_ROTARY_HALVES)
        return fail(GSC_EINVAL, "rotary: unknown pairing %d", pairing);
    if (n < 0 || heads < 1) return fail(GSC_EINVAL, "rotary: bad sizes n=%lld heads=%d", (long long)n, heads);
    if (d < 2 || d > kRotMaxHead || d % 2)
        return fail(GSC_EINVAL, "rotary: d=%d (an even number of 2 to %d channels a head)", d, kRotMaxHead);
    if ((int64_t)heads * d > (1 << 28)) return fail(GSC_EINVAL, "rotary: heads x d = %lld is too large", (long long)heads * d);
    if (D < 1 || D > kRotMaxAxes) return fail(GSC_EINVAL, "rotary: D=%d (1 to %d)", D, kRotMaxAxes);
    if (ldx < (int64_t)heads * d || ldy < (int64_t)heads * d)
        return fail(GSC_EINVAL, "rotary: row strides %lld, %lld below heads x d = %lld", (long long)ldx, (long long)ldy,
                    (long long)heads * d);
    if (!axis_pairs) return fail(GSC_EINVAL, "rotary: null axis_pairs");
    if (!(base >= 1.0) || base > 1e300) return fail(GSC_EINVAL, "rotary: base must be finite and at least 1");
    RotAxes ax;
    ax.D = D;
    ax.log2_base = log2(base);
    int64_t pairs = 0;
    for (int a = 0; a < kRotMaxAxes; ++a) {
        double sc = 1.0;
        if (a < D) {
            if (axis_pairs[a] < 0) return fail(GSC_EINVAL, "rotary: axis_pairs[%d] = %d", a, axis_pairs[a]);
            pairs += axis_pairs[a];
            if (axis_scale) sc = axis_scale[a];
            if (!(fabs(sc) <= 1e6)) return fail(GSC_EINVAL, "rotary: axis_scale[%d] must be at most 1e6 in size", a);
        }
        if (pairs > d / 2) return fail(GSC_EINVAL, "rotary: more than d / 2 = %d pairs", d / 2);
        ax.end[a] = (int)pairs;
        ax.scale[a] = sc / (2.0 * 3.14159265358979323846);
    }
    if (n == 0) return GSC_OK;
    if (!X || !Y || !coords) return fail(GSC_EINVAL, "rotary: null X/Y/coords");
    if (X == Y && ldx != ldy) return fail(GSC_EINVAL, "rotary: in place the two row strides must be equal");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool adj = pairing == GSC_ROTARY_ADJACENT;
    const float sign = inverse ? -1.f : 1.f;
    if (dtype == GSC_BF16) rotary<uint16_t>(X, n, heads, d, ldx, coords, ax, adj, sign, Y, ldy, s);
    else rotary<float>(X, n, heads, d, ldx, coords, ax, adj, sign, Y, ldy, s);
    GSC_LAUNCH_CHECK();
    return GSC_OK;
}

}  // extern "C"
