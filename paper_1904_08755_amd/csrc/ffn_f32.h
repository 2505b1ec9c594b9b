// Tile product of float32 operands for the feed-forward block (ffn.hip): 32 MT x 32 NT outputs per block of
// four waves on v_mfma_f32_16x16x4f32, the operands' next 128 bytes of the reduction in registers
// while the current ones are read from LDS (two stages, one barrier a step).  An operand lies either with the
// reduction along its rows (KC) or across them (MC) and is copied to LDS as it lies; operands
// may start at any float.
#pragma once

#include "row_vec.h"

namespace gsc {

constexpr int kFfnThreads = 256;
constexpr int kFfnRowBytes = 128;               // reduction bytes of a step
constexpr int kFfnBk = kFfnRowBytes / 4;

// One side of a product: `rows` outputs by k reduction elements, element (r, k) at row r and column k of m (KC) or at
// row k and column r (MC).  Rows and reduction elements behind the end read as 0.  SPLIT: the tile's rows
// [0, R / 2) come from m and the others from p2, laid out alike (both from row 0 on, `rows` of each).
struct Side {
    RowMat<const float> m;
    const float* p2;
    int64_t rows;
    int64_t k;
};

// The four floats from `bytes` behind a base that is the same for all lanes, `left` of them valid and the others 0, without
// a branch (the compiler counts the loads in flight).  WHOLE: left is at most 0 or at least 4.
template <bool WHOLE>
__device__ __forceinline__ RowVec<float>::Raw get_f32(const float* base, uint32_t bytes, int64_t left) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, 0x7fffffff, kBufFlags);
    if (WHOLE) return __builtin_amdgcn_raw_buffer_load_b128(rs, left > 0 ? bytes : kBufNone, 0, 0);
    RowVec<float>::Raw r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_raw_buffer_load_b32(rs, e < left ? bytes + 4 * e : kBufNone, 0, 0);
    return r;
}

// A thread's share of a tile of R rows by one step, through registers into LDS.  Its pieces lie `DL` lines apart; SPLIT:
// even ones in the tile's first half, odd ones in the other.  Offsets in bytes from the tile's first element of a step are
// below 2^31 (128 rows of at most 2^20 floats).  WHOLE: no piece ends inside.
template <bool KC, int R, bool SPLIT, bool WHOLE>
struct TileCopy {
    static_assert(!(KC && SPLIT), "only operands across the reduction are split");
    static constexpr int V = 4, BK = kFfnBk, HALVES = SPLIT ? 2 : 1;
    static constexpr int N = R * kFfnRowBytes / 16 / kFfnThreads;      // 16-byte pieces a thread
    static constexpr int PER = KC ? BK / V : R / HALVES / V;           // pieces of a row (KC) or of a reduction element
    static constexpr int DL = kFfnThreads / PER;
    static_assert(N % HALVES == 0 && kFfnThreads % PER == 0, "tile");
    typedef RowVec<float>::Raw Raw;

    RowMat<const float> m;
    const float* p2;
    int line, at;       // first row (KC) or reduction element (MC), and the piece's first element across
    int64_t across;     // MC: elements from `at` to the rows' end (of the half's first one)
    int lim;            // KC: valid lines
    uint32_t off;       // the first piece's offset
    Raw r[N];

    __device__ __forceinline__ void start(const Side& s) {
        line = threadIdx.x / PER;
        at = threadIdx.x % PER * V;
        m = s.m;
        p2 = s.p2;
        lim = (int)(s.rows < R ? s.rows : R);
        across = s.rows - at;
        off = (uint32_t)(KC ? line * m.ld + at : (at >> 5) * m.gs + (at & 31) + line * m.ld) * 4;
    }
    // the step at reduction element k0
    __device__ __forceinline__ void fetch(int64_t k0, int64_t k) {
        const int64_t step = KC ? (k0 >> 5) * m.gs : (k0 >> 7) * m.ts + (k0 & 127) * m.ld;
        const int64_t left = k - k0 - at;
        const int kl = (int)(k - k0 < BK ? k - k0 : BK);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int l = j / HALVES * DL;
            const float* b = (SPLIT && (j & 1) ? p2 : m.p) + step + (int64_t)l * m.ld;
            r[j] = get_f32<WHOLE>(b, off, KC ? (line + l < lim ? left : 0) : (line + l < kl ? across : 0));
        }
    }
    __device__ __forceinline__ void put(uint8_t* lds) const {
        const int c = threadIdx.x % PER;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = line + j / HALVES * DL;
            *reinterpret_cast<uint4*>(lds + place(row, c + (SPLIT && (j & 1) ? PER : 0))) =
                uint4{r[j][0], r[j][1], r[j][2], r[j][3]};
        }
    }
    // Byte of piece c of a line.  KC: lines of 128 bytes, pieces permuted by the row modulo 8, so the
    // eight rows that a read serves together lie in distinct banks.  MC: 64-byte groups permuted by bits 2 and
    // 3 of the reduction element (a lane's q).
    static __device__ __forceinline__ int place(int row, int c) {
        if (KC) return row * kFfnRowBytes + ((c ^ (row & 7)) * 16);
        constexpr int M = R / 16 - 1;
        return row * (R * 4) + (((c >> 2) ^ ((row >> 2) & 3 & M)) * 64) + (c & 3) * 16;
    }
};

// Fragment reads of one wave: operand of 16 rows from row0, reduction elements of group kk (16 of the
// step's 32); lane (i, q) holds row i, elements 4 q .. 4 q + 3, and MFMA s of the four takes the s-th of
// each (the sum does not care which four elements a product takes together).
template <bool KC, int R>
struct Frag {
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
};

// LDS of a block: two stages of both operands.
template <int MT, int NT>
constexpr int ffn_lds() { return 2 * 32 * (MT + NT) * kFfnRowBytes; }

// acc[mi][ni] += the tile's product.  Four waves, (wm, wn) = 2 x 2: wave rows 16 MT wm .., columns
// 16 NT wn .. (SPLIT: half of them from either half of the tile's columns).  The second operand goes
// into the MFMA first, so lane (i, q) gets row 16 mi + i of its rows and four consecutive columns 4 q ..
// of block ni.  LDS may be in use by other waves' earlier reads: starts with a barrier.
// WHOLE: every width is a multiple of four floats.
template <bool AKC, bool BKC, int MT, int NT, bool SPLIT, bool WHOLE>
__device__ __forceinline__ void tile_product(const Side& A, const Side& B, uint8_t* lds, floatx4 (&acc)[MT][NT]) {
    constexpr int RA = 32 * MT, RB = 32 * NT, BK = kFfnBk;
    constexpr int STAGE = (RA + RB) * kFfnRowBytes;
    typedef Frag<AKC, RA> FA;
    typedef Frag<BKC, RB> FB;
    TileCopy<AKC, RA, false, WHOLE> ca;
    TileCopy<BKC, RB, SPLIT, WHOLE> cb;
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
            for (int s = 0; s < 4; ++s)   // (the products of one sum are MT NT instructions apart)
#pragma unroll
                for (int mi = 0; mi < MT; ++mi)
#pragma unroll
                    for (int ni = 0; ni < NT; ++ni)
                        acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[ni][s], a[mi][s], acc[mi][ni], 0, 0, 0);
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

}  // namespace gsc
